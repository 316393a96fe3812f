// Attention of a step's new tokens over the paged 4-bit cache, all pages or selected ones: the kernels without trees.

#include "kv_attention_kernels.h"

namespace ivfpq {

namespace {

template <int D>
int attention_typed(const KvAttnArgs &a, int dtype, const Shape &sh, hipStream_t s) {
  return dtype == IVFPQ_KV_BF16 ? attention_of<D, IVFPQ_KV_BF16, false>(a, sh, s) : attention_of<D, IVFPQ_KV_FP16, false>(a, sh, s);
}

}  // namespace

size_t kv_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_new, int window,
                              int n_select, int64_t width) {
  const Shape s = shape_of(tokens, requests, kv_heads, group, D, max_new, window, n_select, width);
  return s.prefix + s.borders + s.ml + s.o;
}

int launch_kv_attention(KvAttnArgs a, int D, int dtype, int max_new, char *workspace, hipStream_t s) {
  const Shape sh = shape_of(a.tokens, a.requests, a.kv_heads, a.group, D, max_new, a.window, a.selected ? a.n_select : 0,
                            a.width);
  if (!launch_fits(sh.n_wg, sh.tile_rows == 256 || (sh.tile_rows == 128 && D == 256) ? 512 : 256)) {
    set_error("kv_attention: %d workgroups are too many for one launch", sh.n_wg);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  place_workspace(a, sh, workspace);
  switch (D) {
    case 64: return attention_typed<64>(a, dtype, sh, s);
    case 96: return attention_typed<96>(a, dtype, sh, s);
    case 128: return attention_typed<128>(a, dtype, sh, s);
    default: return attention_typed<256>(a, dtype, sh, s);
  }
}

}  // namespace ivfpq

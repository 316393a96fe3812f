// Attention of a step's new tokens over the paged 4-bit cache, all pages or selected ones: the kernels without trees.

#include "kv_attention_kernels.h"

namespace ivfpq {

size_t kv_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_new, int window,
                              int n_select, int64_t width) {
  const Shape s = shape_of(tokens, requests, kv_heads, group, D, max_new, window, n_select, width);
  return s.prefix + s.borders + s.ml + s.o;
}

int launch_kv_attention(KvAttnArgs a, int D, int dtype, int max_new, char *workspace, hipStream_t s) {
  return launch_attention<false>(a, D, dtype, max_new, workspace, s);
}

}  // namespace ivfpq

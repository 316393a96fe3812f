// Attention of drafted tokens over the paged 4-bit cache: what is held before them, and of themselves what their masks say.

#include "kv_attention_kernels.h"

namespace ivfpq {

size_t kv_tree_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_nodes, int window,
                                   int64_t width) {
  const Shape s = shape_of(tokens, requests, kv_heads, group, D, max_nodes, window, 0, width);
  return s.prefix + s.borders + s.ml + s.o;
}

int launch_kv_tree_attention(const KvAttnArgs &a, int D, int dtype, int max_nodes, char *workspace, hipStream_t s) {
  return launch_attention<true>(a, D, dtype, max_nodes, workspace, s);
}

}  // namespace ivfpq

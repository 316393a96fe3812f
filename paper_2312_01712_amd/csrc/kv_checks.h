// Argument checks that the host sides of the paged 4-bit cache share.
#pragma once

#include "kv_internal.h"

namespace ivfpq {

inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline int invalid(const char *fn, const char *what) {
  set_error("%s: %s", fn, what);
  return IVFPQ_ERR_INVALID_ARGUMENT;
}

inline int check_cache(const ivfpq_kv_cache *c, const char *fn) {
  if (!c) return invalid(fn, "cache is NULL");
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) {
    set_error("%s: head_dim = %d, supported are 64, 96, 128 and 256", fn, c->head_dim);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  if (c->kv_heads < 1 || c->kv_heads > 1024) {
    set_error("%s: kv_heads = %d outside [1, 1024]", fn, c->kv_heads);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (c->n_pages < 1 || c->n_pages > ((int64_t)1 << 25)) {
    set_error("%s: n_pages = %lld outside [1, 2^25]", fn, (long long)c->n_pages);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (c->dtype != IVFPQ_KV_BF16 && c->dtype != IVFPQ_KV_FP16) {
    set_error("%s: dtype = %d unknown", fn, c->dtype);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (!c->pages || !c->boxes) return invalid(fn, "NULL array in the cache");
  if (!aligned(c->pages, 16) || !aligned(c->boxes, 16)) return invalid(fn, "pages and boxes must be 16-byte aligned");
  return IVFPQ_OK;
}

inline int check_step(const ivfpq_kv_step *s, const char *fn) {
  if (!s) return invalid(fn, "step is NULL");
  if (s->requests < 0 || s->requests > IVFPQ_KV_MAX_REQUESTS) {
    set_error("%s: requests = %d outside [0, %d]", fn, s->requests, IVFPQ_KV_MAX_REQUESTS);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (s->max_tokens < 0 || s->max_tokens > (1 << 24)) {
    set_error("%s: max_tokens = %d outside [0, 2^24]", fn, s->max_tokens);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (s->table_width < 1 || s->table_width > (1 << 20)) {
    set_error("%s: table_width = %d outside [1, 2^20]", fn, s->table_width);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  return IVFPQ_OK;
}

// The arrays that the kernels read (the workspace sizes do without them).
inline int check_step_arrays(const ivfpq_kv_step *s, const char *fn) {
  if (s->requests > 0 && (!s->kv_lens || !s->table || !s->q_start)) return invalid(fn, "NULL array in the step");
  if (s->max_tokens > 0 && (!s->token_req || !s->positions)) return invalid(fn, "NULL array in the step");
  return IVFPQ_OK;
}

// rows > 1: whether the stride between them is used
inline int check_rows(const void *data, int64_t token_stride, int64_t head_stride, int64_t tokens, int64_t heads, const char *what,
               const char *fn) {
  if (!data || !aligned(data, 16)) {
    set_error("%s: %s is NULL or not 16-byte aligned", fn, what);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if ((tokens > 1 && token_stride % 8) || (heads > 1 && head_stride % 8)) {
    set_error("%s: strides of %s must be multiples of 8 elements", fn, what);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  return IVFPQ_OK;
}

// Whether two rows of D elements share one.
inline bool rows_meet(int64_t token_stride, int64_t head_stride, int64_t tokens, int64_t heads, int D) {
  typedef __int128 wide;  // products of strides and extents
  auto size = [](wide x) { return x < 0 ? -x : x; };
  const wide ts = tokens > 1 ? size(token_stride) : 0, hs = heads > 1 ? size(head_stride) : 0;
  if ((tokens > 1 && ts < D) || (heads > 1 && hs < D)) return true;
  if (tokens < 2 || heads < 2 || ts >= (heads - 1) * hs + D || hs >= (tokens - 1) * ts + D) return false;
  // neither lies within the other: for every distance of heads the tokens that come nearest
  for (int64_t h = 1; h < heads; ++h) {
    const wide t = h * hs / ts;
    if ((t < tokens && h * hs - t * ts < D) || (t + 1 < tokens && (t + 1) * ts - h * hs < D)) return true;
  }
  return false;
}

inline int check_heads(const ivfpq_kv_cache *c, int32_t heads, const char *fn) {
  if (heads < c->kv_heads || heads % c->kv_heads || heads / c->kv_heads > 1024) {
    set_error("%s: heads = %d must be a multiple of kv_heads = %d, 1024 times that at most", fn, heads, c->kv_heads);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  return IVFPQ_OK;
}

inline int check_workspace(const void *p, size_t have, size_t need, const char *fn) {
  if (need > 0 && (!p || !aligned(p, 256) || have < need)) {
    set_error("%s: workspace of %zu bytes, 256-byte aligned, is needed; %zu given", fn, need, p ? have : (size_t)0);
    return IVFPQ_ERR_WORKSPACE;
  }
  return IVFPQ_OK;
}

inline int check_attention(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *a, const char *fn) {
  int rc = check_cache(c, fn);
  if (rc) return rc;
  rc = check_step(s, fn);
  if (rc) return rc;
  if (!a) return invalid(fn, "args is NULL");
  rc = check_heads(c, a->heads, fn);
  if (rc) return rc;
  if (a->n_select < 0 || a->n_select > IVFPQ_KV_MAX_SELECT) {
    set_error("%s: n_select = %d outside [0, %d]", fn, a->n_select, IVFPQ_KV_MAX_SELECT);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (a->window < 0) return invalid(fn, "window must be >= 0");
  if (a->max_new < 1 && s->max_tokens > 0) return invalid(fn, "max_new must be positive");
  // the launch's grid has a workgroup per token, kv head and 16 heads of a group
  const int64_t group = a->heads / c->kv_heads;
  if (((int64_t)s->max_tokens * ((group + 15) / 16) + s->requests) * c->kv_heads > 0x7fffffff ||
      (int64_t)s->max_tokens * group > 0x7fffffff) {
    set_error("%s: max_tokens * heads is too large for one launch", fn);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  return IVFPQ_OK;
}

}  // namespace ivfpq

// C ABI of the paged 4-bit cache (include/ivfpq_kv.h): argument checks and launch arguments; the
// kernels are in kv_plan.hip, kv_append.hip, kv_select.hip and kv_attention.hip.

#include <math.h>

#include "kv_checks.h"

using namespace ivfpq;

extern "C" {

size_t ivfpq_kv_page_bytes(int32_t kv_heads, int32_t head_dim) {
  if (kv_heads < 1 || kv_heads > 1024) return 0;
  if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return 0;
  return (size_t)kv_heads * kv_head_bytes(head_dim);
}

int ivfpq_kv_plan(const ivfpq_kv_step *s, const int32_t *past_lens, const int32_t *new_lens, int32_t *free_pages,
                  int64_t free_capacity, const int64_t *free_state, int64_t *free_state_out, void *stream) {
  const char *fn = "kv_plan";
  int rc = check_step(s, fn);
  if (rc) return rc;
  rc = check_step_arrays(s, fn);
  if (rc) return rc;
  if (!s->q_start || (s->requests > 0 && (!past_lens || !new_lens)) || (s->max_tokens > 0 && !s->slots)) return invalid(fn, "NULL array");
  if (!free_pages || !free_state || !free_state_out) return invalid(fn, "NULL ring of free pages");
  if (free_state == free_state_out) return invalid(fn, "free_state_out must not be free_state");
  if (s->requests > 0 && (s->kv_lens == past_lens || s->kv_lens == new_lens)) return invalid(fn, "kv_lens must not be past_lens or new_lens");
  if (free_capacity < 1 || free_capacity > ((int64_t)1 << 25)) {
    set_error("%s: free_capacity = %lld outside [1, 2^25]", fn, (long long)free_capacity);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  KvPlanArgs a = {};
  a.past = past_lens; a.fresh = new_lens; a.table = s->table; a.free_pages = free_pages; a.kv_lens = s->kv_lens;
  a.q_start = s->q_start; a.token_req = s->token_req; a.positions = s->positions; a.slots = s->slots; a.state = free_state;
  a.state_out = free_state_out; a.capacity = free_capacity; a.requests = s->requests; a.width = s->table_width;
  a.max_tokens = s->max_tokens; a.counts = s->counts;
  return launch_kv_plan(a, static_cast<hipStream_t>(stream));
}

int ivfpq_kv_append(const ivfpq_kv_cache *c, ivfpq_kv_rows k, ivfpq_kv_rows v, const int64_t *slots, int64_t tokens,
                    void *k_rounded, void *v_rounded, void *stream) {
  const char *fn = "kv_append";
  int rc = check_cache(c, fn);
  if (rc) return rc;
  if (tokens < 0 || tokens > (1 << 24)) {
    set_error("%s: tokens = %lld outside [0, 2^24]", fn, (long long)tokens);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (tokens == 0) return IVFPQ_OK;
  rc = check_rows(k.data, k.token_stride, k.head_stride, tokens, c->kv_heads, "k", fn);
  if (rc) return rc;
  rc = check_rows(v.data, v.token_stride, v.head_stride, tokens, c->kv_heads, "v", fn);
  if (rc) return rc;
  if (!slots) return invalid(fn, "slots is NULL");
  if (!aligned(k_rounded, 16) || !aligned(v_rounded, 16)) return invalid(fn, "rounded rows must be 16-byte aligned");
  KvAppendArgs a = {};
  a.pages = static_cast<char *>(c->pages); a.boxes = c->boxes;
  a.k = static_cast<const uint16_t *>(k.data); a.v = static_cast<const uint16_t *>(v.data);
  a.k_rounded = static_cast<uint16_t *>(k_rounded); a.v_rounded = static_cast<uint16_t *>(v_rounded);
  a.slots = slots; a.k_token = k.token_stride; a.k_head = k.head_stride; a.v_token = v.token_stride; a.v_head = v.head_stride;
  a.n_slots = c->n_pages * KV_PAGE; a.tokens = tokens; a.kv_heads = c->kv_heads;
  return launch_kv_append(a, c->head_dim, c->dtype, static_cast<hipStream_t>(stream));
}

size_t ivfpq_kv_select_workspace_bytes(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, int32_t heads) {
  const char *fn = "kv_select_workspace_bytes";
  if (check_cache(c, fn) || check_step(s, fn) || check_heads(c, heads, fn)) return 0;
  return (size_t)s->max_tokens * c->kv_heads * ((s->table_width + 3) & ~3) * sizeof(float);
}

int ivfpq_kv_select(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, ivfpq_kv_rows q, int32_t heads, int32_t n_select,
                    int32_t sinks, int32_t recent, int32_t *d_out, void *d_workspace, size_t workspace_bytes, void *stream) {
  const char *fn = "kv_select";
  int rc = check_cache(c, fn);
  if (rc) return rc;
  rc = check_step(s, fn);
  if (rc) return rc;
  rc = check_heads(c, heads, fn);
  if (rc) return rc;
  if (n_select < 1 || n_select > IVFPQ_KV_MAX_SELECT) {
    set_error("%s: n_select = %d outside [1, %d]", fn, n_select, IVFPQ_KV_MAX_SELECT);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (sinks < 0 || recent < 0 || sinks > n_select || recent > n_select - sinks) {
    set_error("%s: sinks = %d and recent = %d must be >= 0 and n_select = %d together at most", fn, sinks, recent, n_select);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (s->max_tokens == 0) return IVFPQ_OK;
  if ((int64_t)s->max_tokens * c->kv_heads * (s->table_width / 1024 + 1) > 0x7fffffff) {
    set_error("%s: max_tokens * kv_heads * table_width is too large for one launch", fn);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  rc = check_step_arrays(s, fn);
  if (rc) return rc;
  rc = check_rows(q.data, q.token_stride, q.head_stride, s->max_tokens, heads, "q", fn);
  if (rc) return rc;
  if (!d_out) return invalid(fn, "d_out is NULL");
  rc = check_workspace(d_workspace, workspace_bytes, ivfpq_kv_select_workspace_bytes(c, s, heads), fn);
  if (rc) return rc;
  KvSelectArgs a = {};
  a.boxes = c->boxes; a.q = static_cast<const uint16_t *>(q.data); a.table = s->table;
  a.token_req = s->token_req; a.positions = s->positions; a.scores = static_cast<float *>(d_workspace); a.out = d_out;
  a.q_token = q.token_stride; a.q_head = q.head_stride; a.n_pages = c->n_pages; a.kv_heads = c->kv_heads;
  a.group = heads / c->kv_heads; a.requests = s->requests; a.tokens = s->max_tokens; a.width = s->table_width;
  a.score_width = (s->table_width + 3) & ~3; a.n_select = n_select; a.sinks = sinks; a.recent = recent;
  return launch_kv_select(a, c->head_dim, c->dtype, static_cast<hipStream_t>(stream));
}

size_t ivfpq_kv_attention_workspace_bytes(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *a) {
  if (check_attention(c, s, a, "kv_attention_workspace_bytes")) return 0;
  return kv_attention_workspace(s->max_tokens, s->requests, c->kv_heads, a->heads / c->kv_heads, c->head_dim, a->max_new,
                                a->window, a->n_select, s->table_width);
}

int ivfpq_kv_attention(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *x, void *d_workspace,
                       size_t workspace_bytes, void *stream) {
  const char *fn = "kv_attention";
  int rc = check_attention(c, s, x, fn);
  if (rc) return rc;
  if (!isfinite(x->scale)) return invalid(fn, "scale must be finite");
  if (s->max_tokens == 0) return IVFPQ_OK;
  if ((x->selected != nullptr) != (x->n_select > 0)) return invalid(fn, "selected and n_select go together");
  rc = check_step_arrays(s, fn);
  if (rc) return rc;
  rc = check_rows(x->q.data, x->q.token_stride, x->q.head_stride, s->max_tokens, x->heads, "q", fn);
  if (rc) return rc;
  rc = check_rows(x->out, x->out_token_stride, x->out_head_stride, s->max_tokens, x->heads, "out", fn);
  if (rc) return rc;
  if (rows_meet(x->out_token_stride, x->out_head_stride, s->max_tokens, x->heads, c->head_dim)) return invalid(fn, "rows of out overlap");
  const int group = x->heads / c->kv_heads;
  rc = check_workspace(d_workspace, workspace_bytes,
                       kv_attention_workspace(s->max_tokens, s->requests, c->kv_heads, group, c->head_dim, x->max_new,
                                              x->window, x->n_select, s->table_width), fn);
  if (rc) return rc;
  KvAttnArgs a = {};
  a.pages = static_cast<const char *>(c->pages); a.q = static_cast<const uint16_t *>(x->q.data);
  a.out = static_cast<uint16_t *>(x->out); a.lse = x->lse; a.table = s->table; a.q_start = s->q_start; a.kv_lens = s->kv_lens;
  a.token_req = s->token_req; a.positions = s->positions; a.selected = x->selected; a.q_token = x->q.token_stride;
  a.q_head = x->q.head_stride; a.out_token = x->out_token_stride; a.out_head = x->out_head_stride; a.n_pages = c->n_pages;
  a.kv_heads = c->kv_heads; a.group = group; a.requests = s->requests; a.tokens = s->max_tokens; a.width = s->table_width;
  a.n_select = x->n_select; a.window = x->window; 
  // 0 as the smallest number above it: masked keys are -inf, which 0 would turn into NaN
  a.negative = x->scale < 0.0f;
  a.scale2 = fmaxf(fabsf(x->scale) * 1.44269504088896340736f, 1.17549435e-38f);
  return launch_kv_attention(a, c->head_dim, c->dtype, x->max_new, static_cast<char *>(d_workspace),
                             static_cast<hipStream_t>(stream));
}

}  // extern "C"

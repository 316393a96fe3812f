// C ABI of decoding with drafted tokens over the paged 4-bit cache (include/ivfpq_kv.h): argument checks and launch arguments; the
// kernels are in kv_rotate.hip, kv_tree.hip, kv_tree_attention.hip and kv_keep.hip.

#include <math.h>

#include "kv_checks.h"

using namespace ivfpq;

namespace {

int check_tree(const ivfpq_kv_tree *t, const char *fn) {
  if (!t) return invalid(fn, "tree is NULL");
  if (t->max_nodes < 1 || t->max_nodes > IVFPQ_KV_MAX_NODES) {
    set_error("%s: max_nodes = %d outside [1, %d]", fn, t->max_nodes, IVFPQ_KV_MAX_NODES);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (t->window < 0) return invalid(fn, "window must be >= 0");
  return IVFPQ_OK;
}

int check_tree_arrays(const ivfpq_kv_tree *t, const char *fn) {
  if (!t->masks || !t->positions) return invalid(fn, "NULL array in the tree");
  if (!aligned(t->masks, 8)) return invalid(fn, "masks must be 8-byte aligned");
  return IVFPQ_OK;
}

int words_of(const ivfpq_kv_tree *t) { return (t->max_nodes + 63) / 64; }

// What check_attention looks at, with the tree's numbers in the place of the arguments' own.
int check_tree_attention(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *x, const ivfpq_kv_tree *tree,
                         const char *fn) {
  int rc = check_tree(tree, fn);
  if (rc) return rc;
  if (!x) return invalid(fn, "args is NULL");
  ivfpq_kv_attention_args y = *x;
  y.max_new = tree->max_nodes;
  y.window = tree->window;
  rc = check_attention(c, s, &y, fn);
  if (rc) return rc;
  if (x->selected || x->n_select) return invalid(fn, "a tree's tokens look at all pages: selected must be NULL and n_select 0");
  return IVFPQ_OK;
}

}  // namespace

extern "C" {

int ivfpq_kv_rotate(const ivfpq_kv_rotary *r, ivfpq_kv_rows q, int32_t heads, ivfpq_kv_rows k, int32_t kv_heads,
                    const int32_t *positions, int64_t axis_stride, int64_t tokens, ivfpq_kv_out_rows q_out, ivfpq_kv_out_rows k_out,
                    void *stream) {
  const char *fn = "kv_rotate";
  if (!r) return invalid(fn, "rotary is NULL");
  const int D = r->head_dim;
  if (D != 64 && D != 96 && D != 128 && D != 256) {
    set_error("%s: head_dim = %d, supported are 64, 96, 128 and 256", fn, D);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  if (r->turned < 16 || r->turned > D || r->turned % 16) {
    set_error("%s: turned = %d must be a multiple of 16, head_dim = %d at most", fn, r->turned, D);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (r->dtype != IVFPQ_KV_BF16 && r->dtype != IVFPQ_KV_FP16) {
    set_error("%s: dtype = %d unknown", fn, r->dtype);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (r->axes < 1 || r->axes > IVFPQ_KV_MAX_AXES) {
    set_error("%s: axes = %d outside [1, %d]", fn, r->axes, IVFPQ_KV_MAX_AXES);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (heads < 0 || kv_heads < 0 || heads > (1 << 20) || kv_heads > (1 << 20)) return invalid(fn, "heads and kv_heads must be in [0, 2^20]");
  if (tokens < 0 || tokens > (1 << 24)) {
    set_error("%s: tokens = %lld outside [0, 2^24]", fn, (long long)tokens);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if (tokens == 0 || heads + kv_heads == 0) return IVFPQ_OK;
  if (!r->phases || !r->axis || !positions) return invalid(fn, "NULL array");
  int rc;
  if (heads > 0) {
    if ((rc = check_rows(q.data, q.token_stride, q.head_stride, tokens, heads, "q", fn))) return rc;
    if ((rc = check_rows(q_out.data, q_out.token_stride, q_out.head_stride, tokens, heads, "q_out", fn))) return rc;
    if (rows_meet(q_out.token_stride, q_out.head_stride, tokens, heads, D)) return invalid(fn, "rows of q_out overlap");
  }
  if (kv_heads > 0) {
    if ((rc = check_rows(k.data, k.token_stride, k.head_stride, tokens, kv_heads, "k", fn))) return rc;
    if ((rc = check_rows(k_out.data, k_out.token_stride, k_out.head_stride, tokens, kv_heads, "k_out", fn))) return rc;
    if (rows_meet(k_out.token_stride, k_out.head_stride, tokens, kv_heads, D)) return invalid(fn, "rows of k_out overlap");
  }
  KvRotateArgs a = {};
  a.q = static_cast<const uint16_t *>(q.data); a.k = static_cast<const uint16_t *>(k.data);
  a.q_out = static_cast<uint16_t *>(q_out.data); a.k_out = static_cast<uint16_t *>(k_out.data);
  a.positions = positions; a.axis = r->axis; a.phases = r->phases; a.axis_stride = axis_stride; a.tokens = tokens;
  a.q_token = q.token_stride; a.q_head = q.head_stride; a.k_token = k.token_stride; a.k_head = k.head_stride;
  a.qo_token = q_out.token_stride; a.qo_head = q_out.head_stride; a.ko_token = k_out.token_stride; a.ko_head = k_out.head_stride;
  a.heads = heads; a.kv_heads = kv_heads; a.axes = r->axes; a.turned = r->turned; a.dim = D;
  return launch_kv_rotate(a, r->neighbours, r->dtype, static_cast<hipStream_t>(stream));
}

int ivfpq_kv_tree_plan(const ivfpq_kv_step *s, const int32_t *parents, const ivfpq_kv_tree *t, void *stream) {
  const char *fn = "kv_tree_plan";
  int rc = check_step(s, fn);
  if (rc) return rc;
  rc = check_tree(t, fn);
  if (rc) return rc;
  if (s->max_tokens == 0) return IVFPQ_OK;
  rc = check_step_arrays(s, fn);
  if (rc) return rc;
  rc = check_tree_arrays(t, fn);
  if (rc) return rc;
  if (!parents) return invalid(fn, "parents is NULL");
  if (t->positions == s->positions) return invalid(fn, "the tree's positions must not be the step's");
  KvTreeArgs a = {};
  a.q_start = s->q_start; a.positions = s->positions; a.parents = parents; a.masks = t->masks; a.tree_positions = t->positions;
  a.requests = s->requests; a.tokens = s->max_tokens; a.max_nodes = t->max_nodes; a.words = words_of(t); a.window = t->window;
  return launch_kv_tree(a, static_cast<hipStream_t>(stream));
}

size_t ivfpq_kv_tree_attention_workspace_bytes(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *a,
                                               const ivfpq_kv_tree *t) {
  if (check_tree_attention(c, s, a, t, "kv_tree_attention_workspace_bytes")) return 0;
  return kv_tree_attention_workspace(s->max_tokens, s->requests, c->kv_heads, a->heads / c->kv_heads, c->head_dim, t->max_nodes,
                                     t->window, s->table_width);
}

int ivfpq_kv_tree_attention(const ivfpq_kv_cache *c, const ivfpq_kv_step *s, const ivfpq_kv_attention_args *x, const ivfpq_kv_tree *t,
                            void *d_workspace, size_t workspace_bytes, void *stream) {
  const char *fn = "kv_tree_attention";
  int rc = check_tree_attention(c, s, x, t, fn);
  if (rc) return rc;
  if (!isfinite(x->scale)) return invalid(fn, "scale must be finite");
  if (s->max_tokens == 0) return IVFPQ_OK;
  rc = check_step_arrays(s, fn);
  if (rc) return rc;
  rc = check_tree_arrays(t, fn);
  if (rc) return rc;
  rc = check_rows(x->q.data, x->q.token_stride, x->q.head_stride, s->max_tokens, x->heads, "q", fn);
  if (rc) return rc;
  rc = check_rows(x->out, x->out_token_stride, x->out_head_stride, s->max_tokens, x->heads, "out", fn);
  if (rc) return rc;
  if (rows_meet(x->out_token_stride, x->out_head_stride, s->max_tokens, x->heads, c->head_dim)) return invalid(fn, "rows of out overlap");
  const int group = x->heads / c->kv_heads;
  rc = check_workspace(d_workspace, workspace_bytes,
                       kv_tree_attention_workspace(s->max_tokens, s->requests, c->kv_heads, group, c->head_dim, t->max_nodes, t->window,
                                                   s->table_width), fn);
  if (rc) return rc;
  KvAttnArgs a = {};
  a.pages = static_cast<const char *>(c->pages); a.q = static_cast<const uint16_t *>(x->q.data);
  a.out = static_cast<uint16_t *>(x->out); a.lse = x->lse; a.table = s->table; a.q_start = s->q_start; a.kv_lens = s->kv_lens;
  a.token_req = s->token_req; a.positions = s->positions; a.q_token = x->q.token_stride; a.q_head = x->q.head_stride;
  a.out_token = x->out_token_stride; a.out_head = x->out_head_stride; a.n_pages = c->n_pages; a.kv_heads = c->kv_heads;
  a.group = group; a.requests = s->requests; a.tokens = s->max_tokens; a.width = s->table_width; a.window = t->window;
  a.masks = t->masks; a.tree_positions = t->positions; a.words = words_of(t);
  // 0 as the smallest number above it: masked keys are -inf, which 0 would turn into NaN
  a.negative = x->scale < 0.0f;
  a.scale2 = fmaxf(fabsf(x->scale) * 1.44269504088896340736f, 1.17549435e-38f);
  return launch_kv_tree_attention(a, c->head_dim, c->dtype, t->max_nodes, static_cast<char *>(d_workspace),
                                  static_cast<hipStream_t>(stream));
}

int ivfpq_kv_keep(const ivfpq_kv_cache *caches, int32_t n_caches, const ivfpq_kv_step *s, const ivfpq_kv_tree *t,
                  const int32_t *drafted, const int32_t *picked, int32_t *free_pages, int64_t free_capacity, const int64_t *free_state,
                  int64_t *free_state_out, int32_t *lens, int32_t *rows, int32_t *counts, void *stream) {
  const char *fn = "kv_keep";
  if (n_caches < 1 || n_caches > 1024 || !caches) {
    set_error("%s: %d caches, 1 to 1024 are needed", fn, caches ? n_caches : 0);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  int rc;
  for (int i = 0; i < n_caches; ++i) {
    if ((rc = check_cache(caches + i, fn))) return rc;
    if (caches[i].n_pages != caches[0].n_pages || caches[i].kv_heads != caches[0].kv_heads || caches[i].head_dim != caches[0].head_dim ||
        caches[i].dtype != caches[0].dtype)
      return invalid(fn, "the caches must be of one shape and type");
    for (int j = 0; j < i; ++j)
      if (caches[i].pages == caches[j].pages || caches[i].boxes == caches[j].boxes) return invalid(fn, "a cache comes twice");
  }
  if ((rc = check_step(s, fn)) || (rc = check_tree(t, fn))) return rc;
  if (t->window != 0) return invalid(fn, "the tree must be one without a window: its masks name all ancestors");
  if (!free_pages || !free_state || !free_state_out) return invalid(fn, "NULL ring of free pages");
  if (free_state == free_state_out) return invalid(fn, "free_state_out must not be free_state");
  if (free_capacity < 1 || free_capacity > ((int64_t)1 << 25)) {
    set_error("%s: free_capacity = %lld outside [1, 2^25]", fn, (long long)free_capacity);
    return IVFPQ_ERR_INVALID_ARGUMENT;
  }
  if ((rc = check_step_arrays(s, fn))) return rc;
  if (s->requests > 0 && (!lens || !counts)) return invalid(fn, "NULL array");
  if (s->max_tokens > 0) {
    if ((rc = check_tree_arrays(t, fn))) return rc;
    if (!drafted || !picked || !rows || !s->slots) return invalid(fn, "NULL array");
  }
  if (s->requests > 0 && (lens == s->kv_lens || counts == s->kv_lens || lens == counts)) return invalid(fn, "lens and counts must be arrays of their own");
  KvKeepArgs a = {};
  a.q_start = s->q_start; a.kv_lens = s->kv_lens; a.positions = s->positions; a.drafted = drafted; a.picked = picked;
  a.table = s->table; a.slots = s->slots; a.state = free_state; a.masks = t->masks; a.lens = lens; a.rows = rows; a.counts = counts;
  a.free_pages = free_pages; a.state_out = free_state_out; a.n_pages = caches[0].n_pages; a.capacity = free_capacity;
  a.requests = s->requests; a.tokens = s->max_tokens; a.width = s->table_width; a.max_nodes = t->max_nodes; a.words = words_of(t);
  a.kv_heads = caches[0].kv_heads;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if ((rc = launch_kv_accept(a, hs))) return rc;
  for (int at = 0; at < n_caches; at += KEEP_CACHES) {
    a.n_caches = n_caches - at < KEEP_CACHES ? n_caches - at : KEEP_CACHES;
    for (int i = 0; i < a.n_caches; ++i) {
      a.pages[i] = static_cast<char *>(caches[at + i].pages);
      a.boxes[i] = caches[at + i].boxes;
    }
    if ((rc = launch_kv_move(a, caches[0].head_dim, at == 0, hs))) return rc;
  }
  return IVFPQ_OK;
}

int ivfpq_kv_read(const ivfpq_kv_cache *c, const int64_t *slots, int64_t tokens, ivfpq_kv_out_rows k, ivfpq_kv_out_rows v, void *stream) {
  const char *fn = "kv_read";
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
  if (rows_meet(k.token_stride, k.head_stride, tokens, c->kv_heads, c->head_dim) ||
      rows_meet(v.token_stride, v.head_stride, tokens, c->kv_heads, c->head_dim)) return invalid(fn, "rows of k or v overlap");
  if (!slots) return invalid(fn, "slots is NULL");
  KvReadArgs a = {};
  a.pages = static_cast<const char *>(c->pages); a.slots = slots; a.k = static_cast<uint16_t *>(k.data); a.v = static_cast<uint16_t *>(v.data);
  a.k_token = k.token_stride; a.k_head = k.head_stride; a.v_token = v.token_stride; a.v_head = v.head_stride;
  a.n_slots = c->n_pages * KV_PAGE; a.tokens = tokens; a.kv_heads = c->kv_heads;
  return launch_kv_read(a, c->head_dim, c->dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"

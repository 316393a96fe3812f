// Drives the host side of decoding with drafted tokens (csrc/kv_tree_api.hip) with stubs in place of the launchers: refusals, numbers at
// the ends of their ranges, and that what reaches a launcher is what the caller passed.  Pointers are addresses that nothing reads.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "kv_internal.h"

namespace ivfpq {
static char text[512];
static int launched;
static KvAttnArgs attn;
static KvRotateArgs rotated;
static std::vector<KvKeepArgs> moved;
void set_error(const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
}
int hip_fail(hipError_t, const char *) { return IVFPQ_ERR_HIP; }
int launch_kv_rotate(const KvRotateArgs &a, int, int, hipStream_t) { return ++launched, rotated = a, IVFPQ_OK; }
int launch_kv_tree(const KvTreeArgs &, hipStream_t) { return ++launched, IVFPQ_OK; }
int launch_kv_accept(const KvKeepArgs &, hipStream_t) { return ++launched, IVFPQ_OK; }
int launch_kv_move(const KvKeepArgs &a, int, bool ring, hipStream_t) {
  if (ring != moved.empty()) exit(2);
  return ++launched, moved.push_back(a), IVFPQ_OK;
}
int launch_kv_read(const KvReadArgs &, int, int, hipStream_t) { return ++launched, IVFPQ_OK; }
size_t kv_tree_attention_workspace(int64_t tokens, int64_t, int heads, int group, int D, int, int, int64_t) {
  return (size_t)tokens * heads * group * D;
}
int launch_kv_tree_attention(const KvAttnArgs &a, int, int, int, char *, hipStream_t) { return ++launched, attn = a, IVFPQ_OK; }
}  // namespace ivfpq

#define EXPECT(call, want)                                                              \
  do {                                                                                  \
    ivfpq::text[0] = 0;                                                                 \
    const int before = ivfpq::launched, got = (call);                                   \
    if (got != (want) || (got != IVFPQ_OK && (!ivfpq::text[0] || ivfpq::launched != before))) { \
      fprintf(stderr, "line %d: %d, not %d (%s)\n", __LINE__, got, (int)(want), ivfpq::text); \
      exit(1);                                                                          \
    }                                                                                   \
  } while (0)

int main() {
  char *at = reinterpret_cast<char *>(0x100000);
  int32_t *i32 = reinterpret_cast<int32_t *>(at);
  int64_t *i64 = reinterpret_cast<int64_t *>(at);
  uint64_t *u64 = reinterpret_cast<uint64_t *>(at);
  const int BAD = IVFPQ_ERR_INVALID_ARGUMENT;
  const ivfpq_kv_cache cache = {10, 4, 128, IVFPQ_KV_BF16, at, reinterpret_cast<uint16_t *>(at)};
  const ivfpq_kv_step step = {3, 7, 5, i32, i32 + 64, i32, i64, i32, i32, nullptr};
  const ivfpq_kv_rows rows = {at, 4096, 128};
  const ivfpq_kv_out_rows out = {at, 4096, 128};
  // rotate
  ivfpq_kv_rotary rotary = {128, 64, 1, IVFPQ_KV_FP16, 3, u64, i32};
  EXPECT(ivfpq_kv_rotate(&rotary, rows, 32, rows, 8, i32, 9, 7, out, out, nullptr), IVFPQ_OK);
  if (ivfpq::rotated.axis_stride != 9 || ivfpq::rotated.heads != 32 || ivfpq::rotated.kv_heads != 8 || ivfpq::rotated.turned != 64) return 3;
  for (int turned = -16; turned <= 160; turned += 8) {
    rotary.turned = turned;
    EXPECT(ivfpq_kv_rotate(&rotary, rows, 32, rows, 8, i32, 9, 7, out, out, nullptr), turned >= 16 && turned <= 128 && turned % 16 == 0 ? IVFPQ_OK : BAD);
  }
  rotary.turned = 64;
  EXPECT(ivfpq_kv_rotate(&rotary, rows, 0x7fffffff, rows, 0x7fffffff, i32, 9, 7, out, out, nullptr), BAD);
  EXPECT(ivfpq_kv_rotate(&rotary, rows, 0, rows, 8, i32, 0, 1 << 24, out, out, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_rotate(&rotary, rows, 32, rows, 8, i32, 9, INT64_MAX, out, out, nullptr), BAD);
  EXPECT(ivfpq_kv_rotate(&rotary, {at, INT64_MIN, INT64_MIN}, 32, rows, 8, i32, 9, 7, {at, INT64_MIN, 128}, out, nullptr), IVFPQ_OK);
  // trees
  for (int nodes : {-1, 0, 1, 64, 65, 1024, 1025, 0x7fffffff})
    for (int window : {-1, 0, 1, 0x7fffffff}) {
      const ivfpq_kv_tree tree = {nodes, window, u64, i32 + 64};
      const int want = nodes >= 1 && nodes <= 1024 && window >= 0 ? IVFPQ_OK : BAD;
      EXPECT(ivfpq_kv_tree_plan(&step, i32, &tree, nullptr), want);
      ivfpq_kv_attention_args args = {};
      args.q = rows, args.heads = 8, args.scale = -0.5f, args.out = at, args.out_token_stride = 1024, args.out_head_stride = 128;
      const size_t bytes = ivfpq_kv_tree_attention_workspace_bytes(&cache, &step, &args, &tree);
      if ((bytes != 0) != (want == IVFPQ_OK)) return 4;
      EXPECT(ivfpq_kv_tree_attention(&cache, &step, &args, &tree, at, bytes, nullptr), want);
      if (want == IVFPQ_OK && (ivfpq::attn.words != (nodes + 63) / 64 || ivfpq::attn.window != window || !ivfpq::attn.negative)) return 5;
      if (want == IVFPQ_OK) EXPECT(ivfpq_kv_tree_attention(&cache, &step, &args, &tree, at, bytes - 1, nullptr), IVFPQ_ERR_WORKSPACE);
    }
  // keep: any number of caches, 64 a launch, the ring with the first
  const ivfpq_kv_tree tree = {70, 0, u64, i32 + 64};
  for (int n : {1, 2, 63, 64, 65, 128, 1024, 1025}) {
    std::vector<ivfpq_kv_cache> caches(n, cache);
    for (int i = 0; i < n; ++i) caches[i].pages = at + 4096 * i, caches[i].boxes = reinterpret_cast<uint16_t *>(at + 4096 * i);
    ivfpq::moved.clear();
    EXPECT(ivfpq_kv_keep(caches.data(), n, &step, &tree, i32, i32, i32, 10, i64, i64 + 8, i32, i32, i32 + 128, nullptr), n <= 1024 ? IVFPQ_OK : BAD);
    int seen = 0;
    for (const auto &a : ivfpq::moved)
      for (int i = 0; i < a.n_caches; ++i, ++seen)
        if (a.pages[i] != at + 4096 * seen) return 6;
    if (seen != (n <= 1024 ? n : 0)) return 7;
  }
  EXPECT(ivfpq_kv_keep(nullptr, 3, &step, &tree, i32, i32, i32, 10, i64, i64 + 8, i32, i32, i32 + 128, nullptr), BAD);
  ivfpq_kv_step none = {0, 0, 1, nullptr, nullptr, i32, nullptr, nullptr, nullptr, nullptr};
  ivfpq::moved.clear();
  EXPECT(ivfpq_kv_keep(&cache, 1, &none, &tree, nullptr, nullptr, i32, 1, i64, i64 + 8, nullptr, nullptr, nullptr, nullptr), IVFPQ_OK);
  // read
  EXPECT(ivfpq_kv_read(&cache, i64, 9, {at, 512, 128}, {at, 512, 128}, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_read(&cache, i64, 9, {at, 504, 128}, {at, 512, 128}, nullptr), BAD);
  EXPECT(ivfpq_kv_read(&cache, i64, 9, {at, INT64_MAX - 7, 128}, {at, 512, 128}, nullptr), IVFPQ_OK);
  printf("kv_tree_driver: clean\n");
  return 0;
}

// Drives the host side of the paged 4-bit cache's C ABI (csrc/kv_api.hip) with stubs in place of the launchers:
// every refusal, and that what reaches a launcher is what the caller passed.  Pointers are addresses that nothing reads.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "kv_internal.h"

namespace ivfpq {
static char text[512];
static int launched;
static KvAttnArgs seen;
void set_error(const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
}
int hip_fail(hipError_t, const char *) { return IVFPQ_ERR_HIP; }
int launch_kv_plan(const KvPlanArgs &, hipStream_t) { return ++launched, IVFPQ_OK; }
int launch_kv_append(const KvAppendArgs &, int, int, hipStream_t) { return ++launched, IVFPQ_OK; }
int launch_kv_select(const KvSelectArgs &, int, int, hipStream_t) { return ++launched, IVFPQ_OK; }
size_t kv_attention_workspace(int64_t tokens, int64_t, int heads, int group, int D, int, int, int, int64_t) {
  return (size_t)tokens * heads * group * D;
}
int launch_kv_attention(KvAttnArgs a, int, int, int, char *, hipStream_t) { return ++launched, seen = a, IVFPQ_OK; }
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
  const int BAD = IVFPQ_ERR_INVALID_ARGUMENT;
  for (int D = -64; D <= 512; D += 32)
    for (int H : {-1, 0, 1, 8, 1024, 1025}) {
      const bool ok = (D == 64 || D == 96 || D == 128 || D == 256) && H >= 1 && H <= 1024;
      if ((ivfpq_kv_page_bytes(H, D) != 0) != ok) return 1;
    }
  ivfpq_kv_cache cache = {10, 4, 128, IVFPQ_KV_BF16, at, reinterpret_cast<uint16_t *>(at)};
  ivfpq_kv_step step = {3, 7, 5, i32, i32 + 64, i32, i64, i32, i32};
  const ivfpq_kv_rows rows = {at, 4096, 128};
  // plan
  EXPECT(ivfpq_kv_plan(&step, i32, i32, i32, 10, i64, i64 + 8, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_plan(&step, i32, i32, i32, 10, i64, i64, nullptr), BAD);
  EXPECT(ivfpq_kv_plan(&step, i32 + 64, i32, i32, 10, i64, i64 + 8, nullptr), BAD);
  EXPECT(ivfpq_kv_plan(&step, i32, i32, i32, (int64_t)1 << 26, i64, i64 + 8, nullptr), BAD);
  ivfpq_kv_step none = {0, 0, 1, nullptr, nullptr, i32, nullptr, nullptr, nullptr};
  EXPECT(ivfpq_kv_plan(&none, nullptr, nullptr, i32, 1, i64, i64 + 8, nullptr), IVFPQ_OK);
  // append
  EXPECT(ivfpq_kv_append(&cache, rows, rows, i64, 7, nullptr, at, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_append(&cache, rows, rows, i64, (int64_t)1 << 25, nullptr, nullptr, nullptr), BAD);
  // select: the scores of the largest launches stay in 64 bits
  const size_t need = ivfpq_kv_select_workspace_bytes(&cache, &step, 8);
  if (need != (size_t)7 * 4 * 8 * 4) return 1;
  EXPECT(ivfpq_kv_select(&cache, &step, rows, 8, 2, 1, 1, i32, at, need, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_select(&cache, &step, rows, 8, 2, 1, 1, i32, at, need - 1, nullptr), IVFPQ_ERR_WORKSPACE);
  EXPECT(ivfpq_kv_select(&cache, &step, rows, 8, 2, 0x7fffffff, 0x7fffffff, i32, at, need, nullptr), BAD);
  ivfpq_kv_step wide = step;
  wide.max_tokens = 1 << 24, wide.table_width = 1 << 20;
  if (ivfpq_kv_select_workspace_bytes(&cache, &wide, 8) != ((size_t)1 << 24) * 4 * ((size_t)1 << 20) * 4) return 1;
  EXPECT(ivfpq_kv_select(&cache, &wide, rows, 8, 2, 1, 1, i32, at, SIZE_MAX, nullptr), IVFPQ_ERR_UNSUPPORTED);
  // attention
  ivfpq_kv_attention_args a = {rows, 8, 1, 0.5f, 0, nullptr, 0, at, 4096, 128, nullptr};
  const size_t ws = ivfpq_kv_attention_workspace_bytes(&cache, &step, &a);
  EXPECT(ivfpq_kv_attention(&cache, &step, &a, at, ws, nullptr), IVFPQ_OK);
  if (ivfpq::seen.group != 2 || ivfpq::seen.negative || fabsf(ivfpq::seen.scale2 - 0.72134752f) > 1e-6f) return 1;
  a.scale = -0.5f;
  EXPECT(ivfpq_kv_attention(&cache, &step, &a, at, ws, nullptr), IVFPQ_OK);
  if (!ivfpq::seen.negative || !(ivfpq::seen.scale2 > 0.7f)) return 1;
  a.scale = 0.0f;
  EXPECT(ivfpq_kv_attention(&cache, &step, &a, at, ws, nullptr), IVFPQ_OK);
  if (!(ivfpq::seen.scale2 > 0.0f)) return 1;
  a.scale = NAN;
  EXPECT(ivfpq_kv_attention(&cache, &step, &a, at, ws, nullptr), BAD);
  a.scale = 1.0f;
  wide.table_width = 5;
  a.heads = 4096;
  EXPECT(ivfpq_kv_attention(&cache, &wide, &a, at, SIZE_MAX, nullptr), IVFPQ_ERR_UNSUPPORTED);
  a.heads = 8;
  step.max_tokens = 0;
  EXPECT(ivfpq_kv_attention(&cache, &step, &a, nullptr, 0, nullptr), IVFPQ_OK);
  EXPECT(ivfpq_kv_attention(nullptr, nullptr, nullptr, nullptr, 0, nullptr), BAD);
  puts("kv_driver: clean");
  return 0;
}

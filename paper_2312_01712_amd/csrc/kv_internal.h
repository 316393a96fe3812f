// Shared by the kv_*.hip files: launch arguments and the page's layout (include/ivfpq_kv.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ivfpq_kv.h"

namespace ivfpq {

void set_error(const char *fmt, ...);
int hip_fail(hipError_t e, const char *what);

constexpr int KV_PAGE = IVFPQ_KV_PAGE;
// byte offsets within a page and head
constexpr int kv_kscale_at(int D) { return 32 * D; }
constexpr int kv_v_at(int D) { return 34 * D; }
constexpr int kv_vscale_at(int D) { return 66 * D; }
constexpr int kv_head_bytes(int D) { return 68 * D; }

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct KvPlanArgs {
  const int32_t *past, *fresh;
  int32_t *table, *free_pages, *kv_lens, *q_start, *token_req, *positions;
  int32_t *counts;  // [requests] pages of ended requests, or null: every workgroup counts
  int32_t *totals;  // [groups of 16 requests][3] new tokens, pages taken and given; behind the counts, or null
  int64_t *slots;
  const int64_t *state;
  int64_t *state_out, capacity;
  int32_t requests, width, max_tokens, per_group, parts;
};

struct KvAppendArgs {
  char *pages;
  uint16_t *boxes;
  const uint16_t *k, *v;
  uint16_t *k_rounded, *v_rounded;
  const int64_t *slots;
  int64_t k_token, k_head, v_token, v_head, n_slots, tokens;
  int32_t kv_heads;
};

struct KvSelectArgs {
  const uint16_t *boxes, *q;
  const int32_t *table, *token_req, *positions;
  float *scores;  // [tokens][kv_heads][score_width]
  int32_t *out;
  int64_t q_token, q_head, n_pages;
  int32_t kv_heads, group, requests, tokens, width, score_width, n_select, sinks, recent;
};

struct KvAttnArgs {
  const char *pages;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const int32_t *table, *q_start, *kv_lens, *token_req, *positions, *selected;
  int64_t q_token, q_head, out_token, out_head, n_pages;
  int32_t kv_heads, group, requests, tokens, width, n_select, window;
  float scale2;  // |scale| log2(e), above 0
  int32_t negative;  // the scale was below 0
  // workgroups; whether each has a whole unit of rows instead of a share of all units' pages; whether prefix is filled
  int32_t n_wg, whole, scanned;
  int32_t *prefix;   // [requests + 1]: units before each request, where a launch of its own scans them
  int32_t *borders;  // [n_wg][8]: the unit that goes on in the next share
  float *part_ml;    // [2 n_wg][rows of a tile][2]: parts of units that go across borders
  float *part_o;     // [2 n_wg][rows of a tile][D]
};

int launch_kv_plan(const KvPlanArgs &a, hipStream_t s);
int launch_kv_append(const KvAppendArgs &a, int D, int dtype, hipStream_t s);
int launch_kv_select(const KvSelectArgs &a, int D, int dtype, hipStream_t s);
size_t kv_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_new, int window,
                              int n_select, int64_t width);
int launch_kv_attention(KvAttnArgs a, int D, int dtype, int max_new, char *workspace, hipStream_t s);

// A launch may have fewer than 2^32 threads along its grid's first dimension.
inline bool launch_fits(int64_t workgroups, int64_t threads) { return workgroups * threads < (int64_t)1 << 32; }

#define KV_HIP_TRY(expr)                                \
  do {                                                  \
    hipError_t _e = (expr);                             \
    if (_e != hipSuccess) return hip_fail(_e, #expr);   \
  } while (0)

// Element types: the conversions and products of bf16 and fp16 rows.
template <int DTYPE>
struct KvType;

template <>
struct KvType<IVFPQ_KV_BF16> {
  typedef __bf16 elem;
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  static __device__ inline float to_float(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
  static constexpr uint32_t not_finite_bits = 0x7f80;  // sizes from here on are infinite or NaN
  static __device__ inline bool not_finite(uint16_t u) { return (u & 0x7f80) == 0x7f80; }
  static __device__ inline uint32_t pack(float a, float b) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, x2));
  }
  // two held values from byte SEL of w: the low nibble in the low half
  template <int SEL>
  static __device__ inline uint32_t unpack(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
  }
  // two values, divided by the scale and rounded, into byte SEL of w
  template <int SEL>
  static __device__ inline uint32_t round(uint32_t w, uint32_t two, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(x2, two), scale, SEL);
  }
  static __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};

template <>
struct KvType<IVFPQ_KV_FP16> {
  typedef _Float16 elem;
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  static __device__ inline float to_float(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
  static constexpr uint32_t not_finite_bits = 0x7c00;
  static __device__ inline bool not_finite(uint16_t u) { return (u & 0x7c00) == 0x7c00; }
  static __device__ inline uint32_t pack(float a, float b) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, x2));
  }
  template <int SEL>
  static __device__ inline uint32_t unpack(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
  }
  template <int SEL>
  static __device__ inline uint32_t round(uint32_t w, uint32_t two, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(x2, two), scale, SEL);
  }
  static __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};

// 2^(b - 127) of byte I of w, b >= 1
template <int I>
__device__ inline float kv_scale(uint32_t w) {
  return __uint_as_float(I == 3 ? (w >> 1) & 0x7f800000u : ((w >> (8 * I)) & 0xffu) << 23);
}

// Sum over a wavefront's lanes up to and with the own.
__device__ inline int lanes_up_to(int x) {
#define KV_ADD(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false)
  KV_ADD(0x111, 0xf);  // row_shr:1, 2, 4, 8
  KV_ADD(0x112, 0xf);
  KV_ADD(0x114, 0xf);
  KV_ADD(0x118, 0xf);
  KV_ADD(0x142, 0xa);  // row_bcast:15 into rows 1 and 3
  KV_ADD(0x143, 0xc);  // row_bcast:31 into rows 2 and 3
#undef KV_ADD
  return x;
}

}  // namespace ivfpq

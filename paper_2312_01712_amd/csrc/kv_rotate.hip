// Rotary positions: pairs of channels of queries and keys turned by an angle, frequency times position, where every pair
// has its own frequency and its own axis of the position.
//
// Angles are counted in turns, as 64-bit fractions of one: frequency / 2 pi times 2^64, rounded once, times a whole position p, modulo
// 2^64, is off by |p| 2^-65 turns at most (2^-34 at the farthest; in 32 bits a position of 10^6 would leave an angle 0.06 off).  What
// goes to the hardware's sine and cosine, which take turns, is its upper 32 bits (2^-32) as a 32-bit float from -1/2 to 1/2 (2^-26
// turns, 2^-23.3 of an angle, at most).  Sine and cosine themselves were 2^-22.9 off at most of 2^20 places; no bound is documented.

#include "kv_internal.h"

namespace ivfpq {

namespace {

// cosine and sine of position * phase / 2^64 turns
__device__ inline void turn_of(int32_t position, uint64_t phase, float &c, float &s) {
  const uint32_t p = (uint32_t)position, low = (uint32_t)phase;
  uint32_t top = __umulhi(p, low) + p * (uint32_t)(phase >> 32);
  if (position < 0) top -= low;  // p is 2^32 too large
  const float x = (float)(int32_t)top * 0x1p-32f;
  c = __builtin_amdgcn_cosf(x);
  s = __builtin_amdgcn_sinf(x);
}

// A thread has 16 channels (8 pairs, or 16 that are not turned) of every slots-th head of a token, so that it computes its
// sines once for them.  Bound by memory: 9001 tokens of 40 heads of 128, 184 MB, 37 us (5 TB/s); one of 24 heads 2.3 us.
template <int D, int DT, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void kv_rotate_kernel(KvRotateArgs a) {
  constexpr int CHUNKS = D / 16;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const uint32_t chunk = i % CHUNKS, rest = i / CHUNKS, slot = rest % (uint32_t)a.slots;
  const int64_t t = rest / (uint32_t)a.slots;
  if (t >= a.tokens || a.positions[t] < 0) return;
  const int pairs = a.turned / 16;  // chunks that are turned
  const bool turns = (int)chunk < pairs;
  float c[8], s[8];
  if (turns) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t axis = (uint32_t)a.axis[chunk * 8 + j];
      turn_of(a.positions[(axis < (uint32_t)a.axes ? axis : 0) * a.axis_stride + t], a.phases[chunk * 8 + j], c[j], s[j]);
    }
  }
  // the two eights of channels
  const int at0 = turns ? (NEIGHBOURS ? chunk * 16 : chunk * 8) : chunk * 16, at1 = turns && !NEIGHBOURS ? at0 + a.turned / 2 : at0 + 8;
  const int total = a.heads + a.kv_heads;
  for (int h = slot; h < total; h += a.slots) {
    const bool key = h >= a.heads;
    const uint16_t *from = key ? a.k + t * a.k_token + (h - a.heads) * a.k_head : a.q + t * a.q_token + h * a.q_head;
    uint16_t *to = key ? a.k_out + t * a.ko_token + (h - a.heads) * a.ko_head : a.q_out + t * a.qo_token + h * a.qo_head;
    u32x4 x = *reinterpret_cast<const u32x4 *>(from + at0), y = *reinterpret_cast<const u32x4 *>(from + at1);
    if (turns) {
      float u[16], v[16];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u[j] = KvType<DT>::to_float((uint16_t)(x[j >> 1] >> (16 * (j & 1))));
        u[8 + j] = KvType<DT>::to_float((uint16_t)(y[j >> 1] >> (16 * (j & 1))));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int one = NEIGHBOURS ? 2 * j : j, two = NEIGHBOURS ? 2 * j + 1 : 8 + j;
        v[one] = __builtin_fmaf(u[one], c[j], -(u[two] * s[j]));
        v[two] = __builtin_fmaf(u[two], c[j], u[one] * s[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = KvType<DT>::pack(v[2 * j], v[2 * j + 1]);
        y[j] = KvType<DT>::pack(v[8 + 2 * j], v[9 + 2 * j]);
      }
    }
    *reinterpret_cast<u32x4 *>(to + at0) = x;
    *reinterpret_cast<u32x4 *>(to + at1) = y;
  }
}

template <int D, int DT>
void rotate_of(const KvRotateArgs &a, int neighbours, unsigned grid, hipStream_t s) {
  if (neighbours) hipLaunchKernelGGL((kv_rotate_kernel<D, DT, true>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_rotate_kernel<D, DT, false>), dim3(grid), dim3(256), 0, s, a);
}

template <int D>
void rotate_typed(const KvRotateArgs &a, int neighbours, int dtype, unsigned grid, hipStream_t s) {
  if (dtype == IVFPQ_KV_BF16) rotate_of<D, IVFPQ_KV_BF16>(a, neighbours, grid, s);
  else rotate_of<D, IVFPQ_KV_FP16>(a, neighbours, grid, s);
}

}  // namespace

int launch_kv_rotate(const KvRotateArgs &args, int neighbours, int dtype, hipStream_t s) {
  KvRotateArgs a = args;
  const int64_t total = a.heads + (int64_t)a.kv_heads, chunks = a.dim / 16, all = a.tokens * total * chunks;
  // two heads a thread where there are threads enough (40 heads of 128, us, one head a thread, two, four, eight: one token 3.2, 3.3, 3.9,
  // 4.7; 256 4.1, 3.9, 4.6, 5.9; 1024 6.4, 6.0, 6.1, 6.7; 9000 31.7, 30.6, 30.9, 32.2)
  const int64_t per = all >= 65536 ? 2 : 1;
  a.slots = (int32_t)((total + per - 1) / per);
  const int64_t threads = a.tokens * a.slots * chunks;
  if (!launch_fits((threads + 255) / 256, 256)) {
    set_error("kv_rotate: %lld threads are too many for one launch", (long long)threads);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  const unsigned grid = (unsigned)((threads + 255) / 256);
  switch (a.dim) {
    case 64: rotate_typed<64>(a, neighbours, dtype, grid, s); break;
    case 96: rotate_typed<96>(a, neighbours, dtype, grid, s); break;
    case 128: rotate_typed<128>(a, neighbours, dtype, grid, s); break;
    default: rotate_typed<256>(a, neighbours, dtype, grid, s); break;
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

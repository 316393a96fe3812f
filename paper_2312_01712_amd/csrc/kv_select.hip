// Pages for every new token and kv head, by an upper bound on the inner products with the keys of a
// page: the box of the keys takes the place of the per-list boxes of the search path.
//
//   score(page) = max over the query heads of sum_d max(q_d lo_d, q_d hi_d) * 2^e
//               = max over the query heads of (min(q, 0) . lo + max(q, 0) . hi) * 2^e
//
// a product of length 2 D with the box as it lies in memory, [lo | hi].  Queries and corners are 8-bit
// whole numbers, so the products run on the int8 matrix units and the sums are exact in any order.
//
// kv_score_kernel: bound by the boxes, 4 D bytes a page and head; a wavefront has 16 pages, a lane
// 16 channels of one page per step of 64, rounds them to bytes itself (the boxes stay in bf16, where
// they are exact, so that they can grow token by token) and feeds them as they are.
// kv_pick_kernel: one workgroup per token and head finds the n-th largest key by four counts of 8 bits
// and writes the pages above it in order.

#include "kv_internal.h"

namespace ivfpq {

namespace {

constexpr int SCORE_WAVES = 4;
constexpr int SCORE_PAGES = 16 * SCORE_WAVES;  // pages of a workgroup at a time

// Rows of a tile: 16 / GP tokens of one request, GP query heads each (the group's, padded to a power
// of two with its first head).  Groups above 16 heads go through several tiles of one token.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_score_kernel(KvSelectArgs a, int GP, int chunk) {
  constexpr int KSTEPS = 2 * D / 64;
  __shared__ __attribute__((aligned(16))) int8_t rows[16][2 * D + 16];
  __shared__ float tops[16];
  __shared__ int which;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.y;
  const int tpt = GP >= 16 ? 1 : 16 / GP;  // tokens of a tile
  // tile -> request: tiles of request r begin at q_start[r] / tpt + r
  if (tid == 0) {
    int lo = 0, hi = a.requests;  // last r whose first tile is not behind this one
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.q_start[mid] / tpt + mid <= (int)blockIdx.x) lo = mid;
      else hi = mid;
    }
    which = lo;
  }
  __syncthreads();
  const int r = which;
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1];
  const int t0 = q0 + ((int)blockIdx.x - (q0 / tpt + r)) * tpt;
  const int nt = min(tpt, min(q1, a.tokens) - t0);
  if (t0 < max(q0, 0) || nt <= 0) return;
  const int pos_last = a.positions[t0 + nt - 1];
  const int visible = pos_last < 0 ? 0 : min(pos_last / KV_PAGE + 1, a.width);
  const int p0 = blockIdx.z * chunk, p1 = min(p0 + chunk, visible);
  if (p0 >= p1) return;
  const int32_t *table = a.table + (int64_t)r * a.width;

  for (int g0 = 0; g0 < a.group; g0 += 16) {  // once, unless a group has more than 16 heads
    __syncthreads();
    // largest query value of a token and its group: 16 threads a row
    {
      const int row = tid >> 4, part = tid & 15;
      const int t = t0 + min(row / GP, nt - 1);
      float top = 0.0f;
      if (GP < 16 || row == 0) {
        if (row % GP == 0)
          for (int g = 0; g < a.group; ++g)
            for (int c = part; c < D; c += 16) {
              const uint16_t u = a.q[t * a.q_token + (int64_t)(h * a.group + g) * a.q_head + c];
              if (!KvType<DT>::not_finite(u)) top = fmaxf(top, fabsf(KvType<DT>::to_float(u)));
            }
      }
      for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      if (part == 0 && row % GP == 0) tops[row / GP] = top;
    }
    __syncthreads();
    {
      const int row = tid >> 4, part = tid & 15;
      const int tok = min(row / GP, nt - 1);
      int g = g0 + row % GP;
      if (g >= a.group) g = g0;
      float scale = 127.0f * (1.0f / tops[tok]);
      if (!(fabsf(scale) < __builtin_inff())) scale = 0.0f;
      for (int c = part; c < D; c += 16) {
        const uint16_t u = a.q[(int64_t)(t0 + tok) * a.q_token + (int64_t)(h * a.group + g) * a.q_head + c];
        int v = 0;
        if (!KvType<DT>::not_finite(u)) v = (int)rintf(KvType<DT>::to_float(u) * scale);
        rows[row][c] = (int8_t)(v < 0 ? v : 0);
        rows[row][D + c] = (int8_t)(v > 0 ? v : 0);
      }
    }
    __syncthreads();
    i32x4 qa[KSTEPS];
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) qa[s] = *reinterpret_cast<const i32x4 *>(&rows[lane & 15][s * 64 + (lane >> 4) * 16]);

    for (int pb = p0 + wave * 16; pb < p1; pb += SCORE_PAGES) {
      const int col = pb + (lane & 15);
      const int32_t page = col < p1 ? table[col] : -1;
      const bool there = (uint32_t)page < (uint64_t)a.n_pages;
      u32x4 box[KSTEPS][2];
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) {
        box[s][0] = u32x4{0, 0, 0, 0};
        box[s][1] = u32x4{0, 0, 0, 0};
      }
      if (there) {
        const uint16_t *b = a.boxes + ((int64_t)page * a.kv_heads + h) * (2 * D) + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
          box[s][0] = *reinterpret_cast<const u32x4 *>(b + s * 64);
          box[s][1] = *reinterpret_cast<const u32x4 *>(b + s * 64 + 8);
        }
      }
      // exponent of the page's largest corner: the four lanes of a page together
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t w = box[s][j >> 2][j & 3] & 0x7fff7fffu;
          top = max(top, max(w >> 16, w & 0xffffu));
        }
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      int e = (int)(top >> 7);
      e = e < 8 ? 8 : e;
      const float inv = __uint_as_float((uint32_t)(260 - e) << 23);
      i32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) {
        // rounded away from the middle: down in the first half of the row, up in the second
        const bool up = s * 64 + (lane >> 4) * 16 >= D;
        const float f = up ? -inv : inv;
        i32x4 b;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t word = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int at = w * 4 + j;
            const uint32_t two = box[s][at >> 3][(at & 7) >> 1];
            const float x = __uint_as_float((at & 1) ? two & 0xffff0000u : two << 16);
            int v = (int)floorf(x * f);
            v = up ? -v : v;
            word |= ((uint32_t)v & 255u) << (8 * j);
          }
          b[w] = (int)word;
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[s], b, acc, 0, 0, 0);
      }
      // the lane has rows 4 (lane / 16) .. + 3 of its page: the largest of each token's
      const float unit = __uint_as_float((uint32_t)(e - 6) << 23);
      const int first = (lane >> 4) * 4;
      int best[4] = {acc[0], acc[1], acc[2], acc[3]};
      if (GP >= 2) best[0] = max(best[0], best[1]), best[2] = max(best[2], best[3]);
      if (GP >= 4) best[0] = max(best[0], best[2]);
      if (GP >= 8) best[0] = max(best[0], __shfl_xor(best[0], 16));
      if (GP >= 16) best[0] = max(best[0], __shfl_xor(best[0], 32));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = first + i;
        if (row % GP == 0 && row / GP < nt && col < p1) {
          const int t = t0 + row / GP;
          float *to = a.scores + ((int64_t)t * a.kv_heads + h) * a.score_width + col;
          float s = there ? (float)best[i] * unit : -__builtin_inff();
          if (g0 > 0) s = fmaxf(s, *to);
          *to = s;
        }
      }
    }
  }
}

// keys that order like the scores
__device__ inline uint32_t key_of(float s) {
  const uint32_t u = __float_as_uint(s);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int PICK_THREADS = 256;

__global__ __launch_bounds__(PICK_THREADS) void kv_pick_kernel(KvSelectArgs a) {
  __shared__ int counts[256];
  __shared__ int sums[2][PICK_THREADS / 64];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int h = blockIdx.y, n = a.n_select;
  int32_t *out = a.out + (t * a.kv_heads + h) * n;
  const int r = a.token_req[t], pos = a.positions[t];
  // a page number beyond the request's own is never asked for
  const int visible = (uint32_t)r < (uint32_t)a.requests && pos >= 0 ? min(pos / KV_PAGE + 1, a.width) : 0;
  if (visible <= n) {
    for (int i = tid; i < n; i += PICK_THREADS) out[i] = i < visible ? i : -1;
    return;
  }
  const float *scores = a.scores + (t * a.kv_heads + h) * (int64_t)a.score_width;
  auto key_at = [&](int i) -> uint32_t {
    if (i < a.sinks || i >= visible - a.recent) return 0xffffffffu;
    return key_of(scores[i]);
  };
  // the n-th largest key, eight bits at a time
  uint32_t prefix = 0, mask = 0;
  int left = n;  // how many of the keys that share the prefix are wanted
  for (int shift = 24; shift >= 0; shift -= 8) {
    counts[tid] = 0;
    __syncthreads();
    for (int i = tid; i < visible; i += PICK_THREADS) {
      const uint32_t k = key_at(i);
      if ((k & mask) == prefix) atomicAdd(&counts[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // from the largest digit down: the digit at which the count reaches `left`
    if (wave == 0) {
      int c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = counts[255 - (lane * 4 + j)], sum += c[j];
      int before = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(before, d);
        if (lane >= d) before += u;
      }
      before -= sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < left && before + c[j] >= left) found[0] = 255 - (lane * 4 + j), found[1] = left - before;
        before += c[j];
      }
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    mask |= 255u << shift;
    left = found[1];
    __syncthreads();
  }
  // in order: all above the n-th key, and the first `left` of those equal to it
  const int per = (visible + PICK_THREADS - 1) / PICK_THREADS;
  const int i0 = min(tid * per, visible), i1 = min(i0 + per, visible);
  int above = 0, equal = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key_at(i);
    above += k > prefix;
    equal += k == prefix;
  }
  int sa = above, se = equal;
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(sa, d), v = __shfl_up(se, d);
    if (lane >= d) sa += u, se += v;
  }
  if (lane == 63) sums[0][wave] = sa, sums[1][wave] = se;
  __syncthreads();
  for (int w = 0; w < wave; ++w) sa += sums[0][w], se += sums[1][w];
  sa -= above;
  se -= equal;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key_at(i);
    if (k > prefix) {
      out[sa + min(se, left)] = i;
      ++sa;
    } else if (k == prefix) {
      if (se < left) out[sa + se] = i;
      ++se;
    }
  }
}

template <int D>
void score_of(const KvSelectArgs &a, int dtype, dim3 grid, int GP, int chunk, hipStream_t s) {
  if (dtype == IVFPQ_KV_BF16) hipLaunchKernelGGL((kv_score_kernel<D, IVFPQ_KV_BF16>), grid, dim3(256), 0, s, a, GP, chunk);
  else hipLaunchKernelGGL((kv_score_kernel<D, IVFPQ_KV_FP16>), grid, dim3(256), 0, s, a, GP, chunk);
}

}  // namespace

int launch_kv_select(const KvSelectArgs &a, int D, int dtype, hipStream_t s) {
  if (a.requests > 0 && a.width > a.n_select) {
    int GP = 1;
    while (GP < a.group && GP < 16) GP <<= 1;
    const int tpt = GP >= 16 ? 1 : 16 / GP;
    const int64_t tiles = a.tokens / tpt + a.requests;
    // pages of a workgroup: 1024 workgroups and more where there are that many rows, 64 pages at least
    int64_t chunk = (int64_t)a.width * tiles * a.kv_heads / 2048;
    chunk = (chunk + SCORE_PAGES - 1) / SCORE_PAGES * SCORE_PAGES;
    if (chunk < SCORE_PAGES) chunk = SCORE_PAGES;
    if (chunk > 1024) chunk = 1024;
    const dim3 grid((unsigned)tiles, (unsigned)a.kv_heads, (unsigned)((a.width + chunk - 1) / chunk));
    switch (D) {
      case 64: score_of<64>(a, dtype, grid, GP, (int)chunk, s); break;
      case 96: score_of<96>(a, dtype, grid, GP, (int)chunk, s); break;
      case 128: score_of<128>(a, dtype, grid, GP, (int)chunk, s); break;
      default: score_of<256>(a, dtype, grid, GP, (int)chunk, s); break;
    }
    KV_HIP_TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(kv_pick_kernel, dim3((unsigned)a.tokens, (unsigned)a.kv_heads), dim3(PICK_THREADS), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

// Pages for every new token and kv head, by an estimate of the largest inner product with the keys of a
// page: the box of the keys takes the place of the per-list boxes of the search path.
//
//   score(page) = max over the query heads of sum_d max(q_d lo_d, q_d hi_d) * 2^e
//               = max over the query heads of (min(q, 0) . lo + max(q, 0) . hi) * 2^e
//
// a product of length 2 D with the box as it lies in memory, [lo | hi].  Queries and corners are 8-bit
// whole numbers, so the products run on the int8 matrix units and the sums are exact in any order.  Corners are rounded
// outwards, queries to the nearest, so that the score can be below the box's own bound (of normal keys and queries it is in a
// third of the pages); it ranks pages and rules none out.  Of 48 of 1000 pages and 128 of 4000, 99 % are those of the
// unrounded scores.
//
// kv_score_kernel: bound by the boxes, 4 D bytes a page and head; a wavefront has 16 pages, a lane
// 16 channels of one page per step of 64, rounds them to bytes itself (the boxes stay in bf16, where
// they are exact, so that they can grow token by token) and feeds them as they are.  16.8 MB (one token of a
// context of 262 001) 7.6 us, mostly its chain of trips to memory; 60 MB (61 ragged requests) 23 us: 38 % of that is
// vector instructions of the rounding, 12 us the bytes.
// kv_pick_kernel: one workgroup per token and head finds the n-th largest key and writes the pages above it
// in order.

#include "kv_internal.h"

namespace ivfpq {

namespace {

constexpr int SCORE_PAGES = 64;  // pages of a workgroup at a time, 16 a wavefront

// A lane's share of the box of one page: 16 channels of every 64 of [lo | hi].
template <int D>
struct Box {
  u32x4 w[2 * D / 64][2];
};

template <int D>
__device__ inline void load_box(Box<D> &b, const uint16_t *at, bool there) {
#pragma unroll
  for (int s = 0; s < 2 * D / 64; ++s) {
    b.w[s][0] = b.w[s][1] = u32x4{0, 0, 0, 0};
    if (there) {
      b.w[s][0] = *reinterpret_cast<const u32x4 *>(at + s * 64);
      b.w[s][1] = *reinterpret_cast<const u32x4 *>(at + s * 64 + 8);
    }
  }
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The largest whole number that is not above x.
__device__ inline int floor_of(float x) {
  int v;
  asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(v) : "v"(x));
  return v;
}

// Products of 16 rows with the boxes of 16 pages; e: the exponent of a page's unit, plus 6 + 127.  The maxima are taken
// with the other sign, and so are the queries that they meet: down is away from the middle for both halves of the row.
template <int D>
__device__ inline i32x4 box_products(const Box<D> &b, const i32x4 *qa, int lane, int &e) {
  u16x2 most = {0, 0};  // exponent of the page's largest corner: the four lanes of a page together
#pragma unroll
  for (int s = 0; s < 2 * D / 64; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, b.w[s][j >> 2][j & 3] & 0x7fff7fffu));
  uint32_t top = max((uint32_t)most[0], (uint32_t)most[1]);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  e = (int)(top >> 7);
  e = e < 8 ? 8 : e;
  const float inv = __uint_as_float((uint32_t)(260 - e) << 23);
  i32x4 acc = {0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < 2 * D / 64; ++s) {
    const float f = s * 64 + (lane >> 4) * 16 >= D ? -inv : inv;
    i32x4 x;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      int v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = w * 4 + j;
        const uint32_t two = b.w[s][at >> 3][(at & 7) >> 1];
        v[j] = floor_of(__uint_as_float((at & 1) ? two & 0xffff0000u : two << 16) * f);
      }
      const uint32_t low = __builtin_amdgcn_perm((uint32_t)v[1], (uint32_t)v[0], 0x0c0c0400);
      const uint32_t high = __builtin_amdgcn_perm((uint32_t)v[3], (uint32_t)v[2], 0x04000c0c);
      x[w] = (int)(low | high);
    }
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[s], x, acc, 0, 0, 0);
  }
  return acc;
}

// Rows of a tile: `tpt` <= 16 / GP tokens that follow each other, GP query heads each (the group's, padded to a
// power of two with its first head; above 16 heads one token, 16 heads at a time).  Tokens of different
// requests in a tile are scored one request after the other.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_score_kernel(KvSelectArgs a, int GP, int tpt, int chunk) {
  constexpr int KSTEPS = 2 * D / 64, C = D / 16;  // channels that a thread rounds
  __shared__ __attribute__((aligned(16))) int8_t rows[16][2 * D + 16];
  __shared__ float tops[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the heads of a page's boxes lie next to each other: their workgroups run beside each other
  const int tiles = (a.tokens + tpt - 1) / tpt, h = blockIdx.x % a.kv_heads;
  const int tile = blockIdx.x / a.kv_heads % tiles, part_of = blockIdx.x / a.kv_heads / tiles;
  const int t0 = tile * tpt, nt = min(tpt, a.tokens - t0);
  const int row = tid >> 4, part = tid & 15;

  for (int g0 = 0; g0 < a.group; g0 += 16) {  // once, unless a group has more than 16 heads
    i32x4 qa[KSTEPS];
    bool ready = false;
    // a thread's channels of a row: head `first` + row % GP of the row's token, values that are not finite as 0
    auto load_row = [&](int first, float *x) {
      const int tok = min(row / GP, nt - 1);
      int g = first + row % GP;
      if (g >= a.group) g = first;
      const uint32_t *p = reinterpret_cast<const uint32_t *>(a.q + (int64_t)(t0 + tok) * a.q_token +
                                                             (int64_t)(h * a.group + g) * a.q_head + part * C);
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        const uint32_t w = p[c / 2];
        const uint16_t u0 = (uint16_t)w, u1 = (uint16_t)(w >> 16);
        x[c] = KvType<DT>::not_finite(u0) ? 0.0f : KvType<DT>::to_float(u0);
        x[c + 1] = KvType<DT>::not_finite(u1) ? 0.0f : KvType<DT>::to_float(u1);
      }
    };
    // the rows in 8 bits, by the largest value of a token's whole group
    auto round_rows = [&]() {
      float x[C], top = 0.0f;
      if (a.group > 16)
        for (int first = 0; first < a.group; first += 16) {
          load_row(first, x);
#pragma unroll
          for (int c = 0; c < C; ++c) top = fmaxf(top, fabsf(x[c]));
        }
      load_row(g0, x);
#pragma unroll
      for (int c = 0; c < C; ++c) top = fmaxf(top, fabsf(x[c]));
      for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      __syncthreads();
      if (part == 0) tops[row] = top;
      __syncthreads();
      for (int k = row / GP * GP; k < row / GP * GP + GP; ++k) top = fmaxf(top, tops[k]);
      float scale = 127.0f * (1.0f / top);
      if (!(fabsf(scale) < __builtin_inff())) scale = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int v = (int)rintf(x[c] * scale);
        rows[row][part * C + c] = (int8_t)(v < 0 ? v : 0);
        rows[row][D + part * C + c] = (int8_t)(v > 0 ? -v : 0);  // as the maxima: with the other sign
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) qa[s] = *reinterpret_cast<const i32x4 *>(&rows[lane & 15][s * 64 + (lane >> 4) * 16]);
    };

    for (int k0 = 0, k1; k0 < nt; k0 = k1) {  // tokens k0 .. k1 of one request
      const int r = a.token_req[t0 + k0];
      int pos_last = a.positions[t0 + k0];
      for (k1 = k0 + 1; k1 < nt && a.token_req[t0 + k1] == r; ++k1) pos_last = a.positions[t0 + k1];
      const int visible = (uint32_t)r >= (uint32_t)a.requests || pos_last < 0 ? 0 : min(pos_last / KV_PAGE + 1, a.width);
      const int p0 = part_of * chunk, p1 = min(p0 + chunk, visible);
      if (p0 >= p1) continue;
      const int32_t *table = a.table + (int64_t)r * a.width;
      // two tiles of pages ahead: their numbers, and one box
      auto number = [&](int pb) -> int32_t {
        const int col = pb + (lane & 15);
        return col < p1 ? table[col] : -1;
      };
      auto fetch = [&](Box<D> &b, int32_t page) {
        const bool there = (uint32_t)page < (uint64_t)a.n_pages;
        load_box<D>(b, a.boxes + ((int64_t)(there ? page : 0) * a.kv_heads + h) * (2 * D) + (lane >> 4) * 16, there);
      };
      auto finish = [&](const Box<D> &b, int pb, int32_t page) {
        int e;
        const i32x4 acc = box_products<D>(b, qa, lane, e);
        // the lane has rows 4 (lane / 16) .. + 3 of its page: the largest of each token's
        const bool there = (uint32_t)page < (uint64_t)a.n_pages;
        const float unit = __uint_as_float((uint32_t)(e - 6) << 23);
        int best[4] = {acc[0], acc[1], acc[2], acc[3]};
        if (GP >= 2) best[0] = max(best[0], best[1]), best[2] = max(best[2], best[3]);
        if (GP >= 4) best[0] = max(best[0], best[2]);
        if (GP >= 8) best[0] = max(best[0], __shfl_xor(best[0], 16));
        if (GP >= 16) best[0] = max(best[0], __shfl_xor(best[0], 32));
        const int col = pb + (lane & 15);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = (lane >> 4) * 4 + i, k = at / GP;
          if (at % GP == 0 && k >= k0 && k < k1 && col < p1) {
            float *to = a.scores + ((int64_t)(t0 + k) * a.kv_heads + h) * a.score_width + col;
            float s = there ? (float)best[i] * unit : -__builtin_inff();
            if (g0 > 0) s = fmaxf(s, *to);
            *to = s;
          }
        }
      };
      Box<D> even, odd;
      int pb = p0 + wave * 16;
      int32_t page = number(pb), next = number(pb + SCORE_PAGES);
      if (pb < p1) fetch(even, page);
      if (!ready) round_rows();  // while the first boxes are on their way
      ready = true;
      for (; pb < p1; pb += 2 * SCORE_PAGES) {
        const int32_t third = number(pb + 2 * SCORE_PAGES), fourth = number(pb + 3 * SCORE_PAGES);
        fetch(odd, next);
        finish(even, pb, page);
        if (pb + SCORE_PAGES >= p1) break;
        fetch(even, third);
        finish(odd, pb + SCORE_PAGES, next);
        page = third;
        next = fourth;
      }
    }
  }
}

// keys that order like the scores
__device__ inline uint32_t key_of(float s) {
  const uint32_t u = __float_as_uint(s);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int PICK_BINS = 2048;
constexpr int PICK_LAST = 64;  // keys of the last bin that are ranked one by one

// Sum over the workgroup in thread order, up to and with the own; all: of everything.
template <int THREADS>
__device__ inline int block_sum(int x, int *sums, int tid, int &all) {
  const int lane = tid & 63, wave = tid >> 6;
  x = lanes_up_to(x);
  __syncthreads();  // the sums of a call before are read
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  const int before = lanes_up_to(lane < THREADS / 64 ? sums[lane] : 0);
  all = __builtin_amdgcn_readlane(before, THREADS / 64 - 1);
  const int w = __builtin_amdgcn_readfirstlane(wave);
  return w > 0 ? x + __builtin_amdgcn_readlane(before, w - 1) : x;
}

// The columns of one token and head, four a thread and turn.  The n-th largest key: counts of the keys in
// 2048 bins between the smallest and the largest (the scores of a context lie within a few octaves,
// so that bins of equal width spread them); the few keys of the bin that holds it are ranked one by one, many
// are counted again, 11 bits a time.  Up to TURNS * 4 * THREADS columns keep their keys in registers, more
// are read again.  Bound by the latency of its dependent steps (4094 columns: 20.7 us with four counts
// of 8 bits, whose first digit is the same for all).
template <int THREADS, int TURNS>
__global__ __launch_bounds__(THREADS) void kv_pick_kernel(KvSelectArgs a) {
  __shared__ int counts[PICK_BINS];
  __shared__ int sums[THREADS / 64];
  __shared__ uint32_t range[2][THREADS / 64];
  __shared__ int found[3];
  __shared__ uint32_t last_key[PICK_LAST];
  __shared__ int last_col[PICK_LAST], last_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int h = blockIdx.y, n = a.n_select;
  int32_t *out = a.out + (t * a.kv_heads + h) * n;
  const int r = a.token_req[t], pos = a.positions[t];
  // a page number beyond the request's own is never asked for
  const int visible = (uint32_t)r < (uint32_t)a.requests && pos >= 0 ? min(pos / KV_PAGE + 1, a.width) : 0;
  if (visible <= n) {
    for (int i = tid; i < n; i += THREADS) out[i] = i < visible ? i : -1;
    return;
  }
  const float *scores = a.scores + (t * a.kv_heads + h) * (int64_t)a.score_width;
  // columns i .. i + 3 (rows of scores are padded to four); which of them are ranked
  auto load = [&](int i, uint32_t (&k)[4]) {
    const f32x4 s = i < visible ? *reinterpret_cast<const f32x4 *>(scores + i) : f32x4{0, 0, 0, 0};
    for (int j = 0; j < 4; ++j) k[j] = key_of(s[j]);
  };
  auto ranked = [&](int i) { return i >= a.sinks && i < visible - a.recent; };
  uint32_t kept[TURNS][4];
#pragma unroll
  for (int m = 0; m < TURNS; ++m) load((m * THREADS + tid) * 4, kept[m]);
  // every column, in order of turns; f(first column, keys)
  auto each = [&](auto f) {
#pragma unroll
    for (int m = 0; m < TURNS; ++m)
      if (m * THREADS * 4 < visible) f((m * THREADS + tid) * 4, kept[m]);
    for (int b = TURNS * THREADS * 4; b < visible; b += THREADS * 4) {
      uint32_t k[4];
      load(b + tid * 4, k);
      f(b + tid * 4, k);
    }
  };
  for (int b = tid; b < PICK_BINS; b += THREADS) counts[b] = 0;
  if (tid == 0) last_n = 0;
  uint32_t lo = 0xffffffffu, hi = 0;
  each([&](int i, const uint32_t (&k)[4]) {
    for (int j = 0; j < 4; ++j)
      if (ranked(i + j)) lo = min(lo, k[j]), hi = max(hi, k[j]);
  });
  for (int d = 32; d > 0; d >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
  }
  if (lane == 0) range[0][wave] = lo, range[1][wave] = hi;
  __syncthreads();
  for (int w = 0; w < THREADS / 64; ++w) lo = min(lo, range[0][w]), hi = max(hi, range[1][w]);
  // ranked keys above `limit` are in, and those equal to it up to column `limit_col`
  int left = n - a.sinks - a.recent, limit_col = -1, all;
  uint32_t limit = 0xffffffffu;
  while (left > 0) {
    const uint32_t width = hi - lo;
    const int shift = width < PICK_BINS ? 0 : 32 - __clz((int)width) - 11;
    each([&](int i, const uint32_t (&k)[4]) {
      for (int j = 0; j < 4; ++j)
        if (ranked(i + j) && k[j] >= lo && k[j] <= hi) atomicAdd(&counts[(k[j] - lo) >> shift], 1);
    });
    __syncthreads();
    // from the highest bin down: the one at which the count reaches `left`
    constexpr int PER = PICK_BINS / THREADS;
    int c[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) c[j] = counts[PICK_BINS - 1 - (tid * PER + j)], sum += c[j];
    int before = block_sum<THREADS>(sum, sums, tid, all) - sum;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (before < left && before + c[j] >= left)
        found[0] = PICK_BINS - 1 - (tid * PER + j), found[1] = left - before, found[2] = c[j];
      before += c[j];
      counts[PICK_BINS - 1 - (tid * PER + j)] = 0;  // for another turn
    }
    __syncthreads();
    lo += (uint32_t)found[0] << shift;
    hi = min(hi, lo + ((1u << shift) - 1));
    left = found[1];
    const int in_bin = found[2];
    if (in_bin <= PICK_LAST) {
      // all of the bin: in it, the `left`-th by (key down, column up)
      each([&](int i, const uint32_t (&k)[4]) {
        for (int j = 0; j < 4; ++j)
          if (ranked(i + j) && k[j] >= lo && k[j] <= hi) {
            const int at = atomicAdd(&last_n, 1);
            last_key[at] = k[j];
            last_col[at] = i + j;
          }
      });
      __syncthreads();
      if (wave == 0) {
        const uint32_t key = lane < in_bin ? last_key[lane] : 0;
        const int col = lane < in_bin ? last_col[lane] : 0x7fffffff;
        int rank = 0;
        for (int j = 0; j < in_bin; ++j) {
          const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key, j);
          const int c2 = __builtin_amdgcn_readlane(col, j);
          rank += k > key || (k == key && c2 < col);
        }
        if (lane < in_bin && rank == left - 1) found[0] = (int)key, found[1] = col;
      }
      __syncthreads();
      limit = (uint32_t)found[0];
      limit_col = found[1];
      break;
    }
    if (lo == hi) {
      // many equal keys: the first `left` of them, found by counting in order
      int seen = 0;
      each([&](int i, const uint32_t (&k)[4]) {
        int eq = 0;
        for (int j = 0; j < 4; ++j) eq += ranked(i + j) && k[j] == lo;
        int e = seen + block_sum<THREADS>(eq, sums, tid, all) - eq;
        for (int j = 0; j < 4; ++j)
          if (ranked(i + j) && k[j] == lo && ++e == left) found[1] = i + j;
        seen += all;
      });
      __syncthreads();
      limit = lo;
      limit_col = found[1];
      break;
    }
    __syncthreads();  // found is read before it is written again
  }
  int chosen = 0;  // before this turn
  each([&](int i, const uint32_t (&k)[4]) {
    bool in[4];
    int count = 0;
    for (int j = 0; j < 4; ++j) {
      in[j] = i + j < visible && (!ranked(i + j) || (left > 0 && (k[j] > limit || (k[j] == limit && i + j <= limit_col))));
      count += in[j];
    }
    int at = chosen + block_sum<THREADS>(count, sums, tid, all) - count;
    for (int j = 0; j < 4; ++j)
      if (in[j]) out[at++] = i + j;
    chosen += all;
  });
}

template <int D>
void score_of(const KvSelectArgs &a, int dtype, dim3 grid, int GP, int tpt, int chunk, hipStream_t s) {
  if (dtype == IVFPQ_KV_BF16) hipLaunchKernelGGL((kv_score_kernel<D, IVFPQ_KV_BF16>), grid, dim3(256), 0, s, a, GP, tpt, chunk);
  else hipLaunchKernelGGL((kv_score_kernel<D, IVFPQ_KV_FP16>), grid, dim3(256), 0, s, a, GP, tpt, chunk);
}

}  // namespace

int launch_kv_select(const KvSelectArgs &a, int D, int dtype, hipStream_t s) {
  const bool scored = a.requests > 0 && a.width > a.n_select;
  int GP = 1;
  while (GP < a.group && GP < 16) GP <<= 1;
  // one token a tile where a request has one (a tile would have its requests' pages one after the other: 61 requests of
  // 20 000 tokens 25.8 us, four tokens a tile 27.7)
  const int tpt = a.tokens <= a.requests ? 1 : 16 / GP;
  const int64_t tiles = (a.tokens + tpt - 1) / tpt;
  // pages of a workgroup: two turns of its wavefronts (one token of 262 001: 7.5 us, four turns 10.4; 61 ragged requests 22 for
  // both), more where that would be a great many workgroups
  int64_t chunk = 2 * SCORE_PAGES;
  while (chunk < 1024 && tiles * a.kv_heads * ((a.width + chunk - 1) / chunk) > 16384) chunk *= 2;
  const int64_t score_wg = tiles * a.kv_heads * ((a.width + chunk - 1) / chunk);
  const int pick_threads = a.width <= 1024 ? 256 : 1024;
  if ((scored && !launch_fits(score_wg, 256)) || !launch_fits(a.tokens, pick_threads)) {
    set_error("kv_select: %d tokens of %d kv heads and %d columns are too many for one launch", a.tokens, a.kv_heads, a.width);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  if (scored) {
    const dim3 grid((unsigned)score_wg);
    switch (D) {
      case 64: score_of<64>(a, dtype, grid, GP, tpt, (int)chunk, s); break;
      case 96: score_of<96>(a, dtype, grid, GP, tpt, (int)chunk, s); break;
      case 128: score_of<128>(a, dtype, grid, GP, tpt, (int)chunk, s); break;
      default: score_of<256>(a, dtype, grid, GP, tpt, (int)chunk, s); break;
    }
    KV_HIP_TRY(hipGetLastError());
  }
  // threads by the columns that their registers hold (700 columns: 25.4 us both launches, 1024 threads 26.2; 3200: 21.0, 256
  // threads 25.3)
  const dim3 grid((unsigned)a.tokens, (unsigned)a.kv_heads);
  if (a.width <= 1024) hipLaunchKernelGGL((kv_pick_kernel<256, 1>), grid, dim3(pick_threads), 0, s, a);
  else if (a.width <= 4096) hipLaunchKernelGGL((kv_pick_kernel<1024, 1>), grid, dim3(pick_threads), 0, s, a);
  else hipLaunchKernelGGL((kv_pick_kernel<1024, 4>), grid, dim3(pick_threads), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

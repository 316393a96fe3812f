// Tokens that are held already: those that stay of a step's drafted ones move together, the boxes of their pages are made again,
// pages behind them go back; and held tokens read back as rows.

#include "kv_internal.h"

namespace ivfpq {

namespace {

// eight codes, the first channel lowest, as values of the cache's type
template <int DT>
__device__ inline u32x4 held_row(uint32_t w, uint32_t b) {
  const float scale = __uint_as_float(b << 23);
  u32x4 r;
  r[0] = KvType<DT>::template unpack<0>(w, scale);
  r[1] = KvType<DT>::template unpack<1>(w, scale);
  r[2] = KvType<DT>::template unpack<2>(w, scale);
  r[3] = KvType<DT>::template unpack<3>(w, scale);
  return r;
}

// Byte e (below 68 D / 64) of the token at `place` of a page and head.
template <int D>
__device__ inline int byte_at(int e, int place) {
  const int lane = ((place >> 2) & 3) * 16, word = (place >> 4) * 4 + (place & 3);
  if (e < D / 2) return place * (D / 2) + e;
  e -= D / 2;
  if (e < D / 32) return kv_kscale_at(D) + ((place & 15) * (D / 32) + e) * 4 + (place >> 4);
  e -= D / 32;
  if (e < D / 2) return kv_v_at(D) + (e >> 4) * 1024 + (lane + (e & 15)) * 16 + word;
  e -= D / 2;
  return kv_vscale_at(D) + e * 64 + lane + word;
}

// Orders a wavefront's accesses to memory that other lanes of it have written or will write.
__device__ inline void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  __builtin_amdgcn_wave_barrier();
}

// Pages of request r behind what stays, behind those that earlier requests give back; by the whole workgroup.
__device__ inline void give_back(const KvKeepArgs &a, int r, int tid) {
  __shared__ int64_t sums[4];
  const int lane = tid & 63, wave = tid >> 6;
  const int64_t head = a.state[0], tail = a.state[1];
  const int own = r < a.requests ? a.counts[r] : 0;
  const bool last = r >= a.requests - 1;
  if (own == 0 && !last) return;
  int64_t before = 0;
  for (int b = tid; b < r; b += 256) before += a.counts[b];
  for (int d = 32; d > 0; d >>= 1) before += __shfl_xor(before, d);
  if (lane == 0) sums[wave] = before;
  __syncthreads();
  before = sums[0] + sums[1] + sums[2] + sums[3];
  const int64_t avail = tail > head ? min(tail - head, a.capacity) : 0, room = a.capacity - avail;
  if (last && tid == 0) {
    a.state_out[0] = head;
    a.state_out[1] = tail + min(before + own, room);
    a.state_out[2] = a.state[2];
  }
  if (own == 0 || wave != 0) return;
  int64_t tail_at = tail % a.capacity;
  if (tail_at < 0) tail_at += a.capacity;
  const int from = (int)(((int64_t)a.lens[r] + KV_PAGE - 1) / KV_PAGE);
  const int to = min((int)(((int64_t)a.kv_lens[r] + KV_PAGE - 1) / KV_PAGE), a.width);
  for (int c = from; c < to; c += 64) {
    const int page = c + lane < to ? a.table[(int64_t)r * a.width + c + lane] : -1;
    const uint64_t there = __ballot((uint32_t)page < (uint64_t)a.n_pages);
    const int64_t at = before + __builtin_popcountll(there & ((1ull << lane) - 1));
    if ((there >> lane & 1) && at < room) a.free_pages[(tail_at + at) % a.capacity] = page;
    before += __builtin_popcountll(there);
  }
}

// A wavefront has one request, kv head and cache.  What stays moves to lower slots in the order of tokens, four at a time: what a
// later one comes from lies behind everything written.  Keys are 4-bit codes still, so the boxes that they give are those that
// appending only the tokens that stay would have given.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_move_kernel(KvKeepArgs a, int ring) {
  constexpr int BYTES = 68 * D / 64, TRIPS = (BYTES + 63) / 64, AHEAD = 4;
  constexpr int OCT = D / 8, TOKENS = 64 / OCT;  // lanes of a token's keys, tokens at a time
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x;
  if (ring && blockIdx.y == 0 && blockIdx.z == 0) give_back(a, r, tid);
  const int h = blockIdx.y * 4 + wave;
  if (r >= a.requests || h >= a.kv_heads) return;
  const int t0 = min(max(a.q_start[r], 0), a.tokens), n = min(a.q_start[r + 1], a.tokens) - t0;
  if (n <= 0) return;
  const int past = max(a.positions[t0], 0), stays = a.lens[r], kept = min(stays - past, n);
  if (kept <= 0 || kept == n) return;  // all of them stay where they are
  char *pages = a.pages[blockIdx.z] + (int64_t)h * kv_head_bytes(D);
  const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D), n_slots = a.n_pages * KV_PAGE;

  for (int b = 0; b < kept; b += AHEAD) {
    int64_t from[AHEAD], to[AHEAD];
    bool any = false;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = min(b + j, kept - 1), row = a.rows[t0 + i];
      from[j] = row >= 0 && row < a.tokens ? a.slots[row] : -1;
      to[j] = a.slots[t0 + i];
      if (b + j >= kept || from[j] == to[j] || from[j] < 0 || from[j] >= n_slots || to[j] >= n_slots) to[j] = -1;
      any = any || to[j] >= 0;
    }
    if (!any) continue;
    uint8_t x[AHEAD][TRIPS];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int m = 0; m < TRIPS; ++m)
        if (to[j] >= 0 && m * 64 + lane < BYTES)
          x[j][m] = *reinterpret_cast<const uint8_t *>(pages + from[j] / KV_PAGE * page_bytes + byte_at<D>(m * 64 + lane, (int)(from[j] % KV_PAGE)));
    wave_fence();
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int m = 0; m < TRIPS; ++m)
        if (to[j] >= 0 && m * 64 + lane < BYTES)
          *reinterpret_cast<uint8_t *>(pages + to[j] / KV_PAGE * page_bytes + byte_at<D>(m * 64 + lane, (int)(to[j] % KV_PAGE))) = x[j][m];
    wave_fence();
  }

  // the boxes of the pages that the tokens which stay lie in
  const int sub = lane / OCT, oct = lane % OCT;
  for (int c = past / KV_PAGE; c * (int64_t)KV_PAGE < stays && c < a.width; ++c) {
    const int page = a.table[(int64_t)r * a.width + c];
    if ((uint32_t)page >= (uint64_t)a.n_pages) continue;
    const char *at = pages + page * page_bytes;
    const int count = min(KV_PAGE, stays - c * KV_PAGE);
    float low[8], high[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) low[j] = __builtin_inff(), high[j] = -__builtin_inff();
#pragma unroll 4
    for (int t = sub < TOKENS ? sub : count; t < count; t += TOKENS) {
      const uint32_t codes = *reinterpret_cast<const uint32_t *>(at + t * (D / 2) + oct * 4);
      uint32_t b = *reinterpret_cast<const uint8_t *>(at + kv_kscale_at(D) + ((t & 15) * (D / 32) + oct / 4) * 4 + (t >> 4));
      if (b == 255) b = 1;  // a token that is no number: its codes are 0
      const u32x4 x = held_row<DT>(codes, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = KvType<DT>::to_float((uint16_t)(x[j >> 1] >> (16 * (j & 1))));
        low[j] = fminf(low[j], v);
        high[j] = fmaxf(high[j], v);
      }
    }
    u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float l = low[j], u = high[j];
#pragma unroll
      for (int q = 1; q < TOKENS; ++q) {
        l = fminf(l, __shfl(low[j], oct + q * OCT));
        u = fmaxf(u, __shfl(high[j], oct + q * OCT));
      }
      lo[j >> 1] |= (__float_as_uint(l) >> 16) << (16 * (j & 1));  // exact: two significant bits
      hi[j >> 1] |= (__float_as_uint(u) >> 16) << (16 * (j & 1));
    }
    if (lane < OCT) {
      uint16_t *box = a.boxes[blockIdx.z] + (((int64_t)page * a.kv_heads + h) * 2) * D + oct * 8;
      *reinterpret_cast<u32x4 *>(box) = lo;
      *reinterpret_cast<u32x4 *>(box + D) = hi;
    }
  }
}

// D / 8 lanes have a token and head, eight channels each.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a) {
  constexpr int OCT = D / 8;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, rest = i / OCT;
  const int oct = i % OCT, h = rest % (uint32_t)a.kv_heads;
  const int64_t t = rest / (uint32_t)a.kv_heads;
  if (t >= a.tokens) return;
  const int64_t slot = a.slots[t];
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (slot >= 0 && slot < a.n_slots) {
    const int place = (int)(slot % KV_PAGE), group = oct >> 2;
    const char *at = a.pages + (slot / KV_PAGE * a.kv_heads + h) * (int64_t)kv_head_bytes(D);
    const int lane = ((place >> 2) & 3) * 16, word = (place >> 4) * 4 + (place & 3);
    const uint32_t kc = *reinterpret_cast<const uint32_t *>(at + place * (D / 2) + oct * 4);
    const uint32_t kb = *reinterpret_cast<const uint8_t *>(at + kv_kscale_at(D) + ((place & 15) * (D / 32) + group) * 4 + (place >> 4));
    const uint32_t vb = *reinterpret_cast<const uint8_t *>(at + kv_vscale_at(D) + group * 64 + lane + word);
    const char *vp = at + kv_v_at(D) + group * 1024 + (lane + (oct & 1) * 8) * 16 + word;
    uint32_t vc = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) vc |= ((uint32_t)*reinterpret_cast<const uint8_t *>(vp + j * 16) >> (2 * (oct & 2)) & 15u) << (4 * j);
    k = kb == 255 ? u32x4{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu} : held_row<DT>(kc, kb);
    v = held_row<DT>(vc, vb);
  }
  *reinterpret_cast<u32x4 *>(a.k + t * a.k_token + h * a.k_head + oct * 8) = k;
  *reinterpret_cast<u32x4 *>(a.v + t * a.v_token + h * a.v_head + oct * 8) = v;
}

template <int D>
int read_of(const KvReadArgs &a, int dtype, hipStream_t s) {
  const int64_t groups = (a.tokens * a.kv_heads * (D / 8) + 255) / 256;
  if (!launch_fits(groups, 256)) {
    set_error("kv_read: %lld workgroups are too many for one launch", (long long)groups);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  if (dtype == IVFPQ_KV_BF16) hipLaunchKernelGGL((kv_read_kernel<D, IVFPQ_KV_BF16>), dim3((unsigned)groups), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_read_kernel<D, IVFPQ_KV_FP16>), dim3((unsigned)groups), dim3(256), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

template <int D>
void move_of(const KvKeepArgs &a, int dtype, int ring, hipStream_t s) {
  const dim3 grid((unsigned)(a.requests > 0 ? a.requests : 1), (unsigned)((a.kv_heads + 3) / 4), (unsigned)a.n_caches);
  if (dtype == IVFPQ_KV_BF16) hipLaunchKernelGGL((kv_move_kernel<D, IVFPQ_KV_BF16>), grid, dim3(256), 0, s, a, ring);
  else hipLaunchKernelGGL((kv_move_kernel<D, IVFPQ_KV_FP16>), grid, dim3(256), 0, s, a, ring);
}

}  // namespace

int launch_kv_move(const KvKeepArgs &a, int D, int dtype, bool ring, hipStream_t s) {
  switch (D) {
    case 64: move_of<64>(a, dtype, ring, s); break;
    case 96: move_of<96>(a, dtype, ring, s); break;
    case 128: move_of<128>(a, dtype, ring, s); break;
    default: move_of<256>(a, dtype, ring, s); break;
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

int launch_kv_read(const KvReadArgs &a, int D, int dtype, hipStream_t s) {
  switch (D) {
    case 64: return read_of<64>(a, dtype, s);
    case 96: return read_of<96>(a, dtype, s);
    case 128: return read_of<128>(a, dtype, s);
    default: return read_of<256>(a, dtype, s);
  }
}

}  // namespace ivfpq

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

// Byte e (below 68 D / 64) of the token at `place` of a page and head lies at byte_base(e) + byte_place(kind of e, place).
template <int D>
__device__ inline int byte_kind(int e) { return e < D / 2 ? 0 : e < D / 2 + D / 32 ? 1 : e < D + D / 32 ? 2 : 3; }
template <int D>
__device__ inline int byte_base(int e) {
  const int kind = byte_kind<D>(e);
  if (kind == 0) return e;
  e -= D / 2;
  if (kind == 1) return kv_kscale_at(D) + e * 4;
  e -= D / 32;
  if (kind == 2) return kv_v_at(D) + (e >> 4) * 1024 + (e & 15) * 16;
  return kv_vscale_at(D) + (e - D / 2) * 64;
}
template <int D>
__device__ inline int byte_place(int kind, int place) {
  const int word = (place >> 4) * 4 + (place & 3), quad = (place >> 2) & 3;
  return kind == 0 ? place * (D / 2) : kind == 1 ? (place & 15) * (D / 8) + (place >> 4) : kind == 2 ? quad * 256 + word : quad * 16 + word;
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

// Eight channels' smallest and largest values so far.
struct Box {
  float low[8], high[8];

  __device__ inline void clear() {
#pragma unroll
    for (int j = 0; j < 8; ++j) low[j] = __builtin_inff(), high[j] = -__builtin_inff();
  }

  // two tokens' codes and scales
  __device__ inline void add(uint32_t w0, uint32_t b0, uint32_t w1, uint32_t b1) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    // (255: a token that is no number, its codes are 0)
    const float s0 = __uint_as_float((b0 == 255 ? 1 : b0) << 23), s1 = __uint_as_float((b1 == 255 ? 1 : b1) << 23);
    auto pair = [&](f32x2 x, f32x2 y, int j) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        low[j + i] = fminf(fminf(low[j + i], x[i]), y[i]);
        high[j + i] = fmaxf(fmaxf(high[j + i], x[i]), y[i]);
      }
    };
    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w0, s0, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w1, s1, 0), 0);
    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w0, s0, 1), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w1, s1, 1), 2);
    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w0, s0, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w1, s1, 2), 4);
    pair(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w0, s0, 3), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w1, s1, 3), 6);
  }
};

// A wavefront has one request, kv head and cache.  First the boxes, from where the tokens that stay lie before they move (keys are
// 4-bit codes still, so these are the boxes that appending only them would have given); then what stays moves to lower slots in the
// order of tokens, four at a time: what a later one comes from lies behind everything written.  SMALL: no request has more than 64
// new tokens, a lane each, which takes three trips to memory before the first write.  Bound by these trips: 48 requests of up to
// 64 drafted tokens, 8 heads of 128, 28 caches, 43 MB, 23 us (the boxes behind the moves, a value at a time, 34);
// one request, 4 caches, 6.4 (the moves behind the boxes, the ring by the first workgroups, 6.7).
template <int D, bool SMALL>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 96 ? 4 : 7))) void kv_move_kernel(KvKeepArgs a) {
  constexpr int BYTES = 68 * D / 64, TRIPS = (BYTES + 63) / 64, AHEAD = 4;
  constexpr int OCT = D / 8, TOKENS = 64 / OCT, TRIP = 8;  // lanes of a token's keys, tokens at a time, of which so many on their way
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x;
  if ((int)blockIdx.z == a.n_caches) {  // behind the caches: the ring
    if (blockIdx.y == 0) give_back(a, r, tid);
    return;
  }
  const int h = blockIdx.y * 4 + wave;
  if (r >= a.requests || h >= a.kv_heads) return;
  const int t0 = min(max(a.q_start[r], 0), a.tokens), n = min(a.q_start[r + 1], a.tokens) - t0, kv = a.kv_lens[r], stays = a.lens[r];
  if (n <= 0) return;
  // (where the table's width has cut the request its length does not say where its new tokens begin)
  const int past = kv < a.width * (int64_t)KV_PAGE ? max(kv - n, 0) : max(a.positions[t0], 0);
  const int kept = min(stays - past, n);
  if (kept < 0 || kept == n) return;  // all of them stay where they are
  // (none of them: only the box is made, of what was held; `end` is then that of a token which is not used)
  const int end = max(kept, 1) - 1;
  char *pages = a.pages[blockIdx.z] + (int64_t)h * kv_head_bytes(D);
  const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
  const uint64_t n_slots = a.n_pages * KV_PAGE;
  const int first_column = past / KV_PAGE, end_column = min((int)(((int64_t)stays + KV_PAGE - 1) / KV_PAGE), a.width);

  // where token i of those that stay comes from, and goes to
  int64_t own_from = -1, own_to = -1;
  int own_page = -1, in_place = kept;  // the first of them that moves
  if constexpr (SMALL) {
    const int row = a.rows[t0 + min(lane, end)] - t0;
    own_to = lane < n ? a.slots[t0 + lane] : -1;
    own_page = first_column + lane < end_column ? a.table[(int64_t)r * a.width + first_column + lane] : -1;
    own_from = __shfl(own_to, row & 63);
    const uint64_t moved = __ballot(lane < kept && row != lane);
    if (moved) in_place = __builtin_ctzll(moved);
  } else {
    for (int b = 0; b < kept; b += 64) {
      const uint64_t moved = __ballot(b + lane < kept && a.rows[t0 + min(b + lane, end)] - t0 != b + lane);
      if (moved) {
        in_place = b + __builtin_ctzll(moved);
        break;
      }
    }
  }
  auto uniform64 = [](int64_t x, int i) -> int64_t {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, i), hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), i);
    return (int64_t)((uint64_t)hi << 32 | lo);
  };
  auto target = [&](int i) -> int64_t { return SMALL ? uniform64(own_to, i & 63) : uniform64(a.slots[t0 + i], 0); };
  auto source = [&](int i) -> int64_t {  // i has a row, and both slots are in the cache; otherwise where it goes to
    int64_t from = -1;
    if constexpr (SMALL) {
      from = uniform64(own_from, i & 63);
    } else {
      const int row = __builtin_amdgcn_readfirstlane(a.rows[t0 + i]);
      if (row >= 0 && row < a.tokens) from = uniform64(a.slots[row], 0);
    }
    const int64_t to = target(i);
    return (uint64_t)from < n_slots && (uint64_t)to < n_slots ? from : to;
  };

  // four tokens' bytes, from where they are to where they go; the first four are on their way while the boxes are made
  int kind[TRIPS], base[TRIPS];
#pragma unroll
  for (int m = 0; m < TRIPS; ++m) kind[m] = byte_kind<D>(m * 64 + lane), base[m] = byte_base<D>(m * 64 + lane);
  uint8_t x[AHEAD][TRIPS];
  int64_t to[AHEAD];
  auto load = [&](int i0) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = min(i0 + j, end);
      const int64_t from = source(i);
      to[j] = target(i);
      if (i0 + j >= kept || from == to[j]) to[j] = -1;  // (also where one of the two is nowhere)
      if (to[j] < 0) continue;
      const char *at = pages + (from >> 6) * page_bytes;
#pragma unroll
      for (int m = 0; m < TRIPS; ++m)
        if (m * 64 + lane < BYTES) x[j][m] = *reinterpret_cast<const uint8_t *>(at + base[m] + byte_place<D>(kind[m], (int)from & 63));
    }
  };
  auto store = [&]() {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (to[j] < 0) continue;
      char *at = pages + (to[j] >> 6) * page_bytes;
#pragma unroll
      for (int m = 0; m < TRIPS; ++m)
        if (m * 64 + lane < BYTES) *reinterpret_cast<uint8_t *>(at + base[m] + byte_place<D>(kind[m], (int)to[j] & 63)) = x[j][m];
    }
  };
  load(in_place);

  const int sub = lane / OCT, oct = lane % OCT;
  for (int c = first_column; c < end_column; ++c) {
    const int page = SMALL ? __builtin_amdgcn_readlane(own_page, (c - first_column) & 63) : __builtin_amdgcn_readfirstlane(a.table[(int64_t)r * a.width + c]);
    if ((uint32_t)page >= (uint64_t)a.n_pages) continue;
    Box box;
    box.clear();
    auto keys = [&](const char *at, int place, uint32_t &w, uint32_t &b) {
      w = *reinterpret_cast<const uint32_t *>(at + place * (D / 2) + oct * 4);
      b = *reinterpret_cast<const uint8_t *>(at + kv_kscale_at(D) + ((place & 15) * (D / 32) + oct / 4) * 4 + (place >> 4));
    };
    // tokens that lie in the page already
    const char *at = pages + page * page_bytes;
    const int count = min(KV_PAGE, min(stays, past + in_place) - c * KV_PAGE);
    for (int p0 = 0; p0 < count; p0 += TRIP * TOKENS) {
      uint32_t w[TRIP], b[TRIP];
#pragma unroll
      for (int i = 0; i < TRIP; ++i) keys(at, min(p0 + i * TOKENS + min(sub, TOKENS - 1), count - 1), w[i], b[i]);
#pragma unroll
      for (int i = 0; i < TRIP; i += 2) box.add(w[i], b[i], w[i + 1], b[i + 1]);
    }
    // and those that will
    const int last = min(kept, (c + 1) * KV_PAGE - past);
    for (int i = max(in_place, c * KV_PAGE - past); i < last; i += 2) {
      uint32_t w[2], b[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t slot = source(min(i + j, last - 1));
        if ((uint64_t)slot < n_slots) keys(pages + (slot >> 6) * page_bytes, (int)slot & 63, w[j], b[j]);
        else keys(at, 0, w[j], b[j]);  // (nowhere: not in a page that is there)
      }
      box.add(w[0], b[0], w[1], b[1]);
    }
    u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float l = box.low[j], u = box.high[j];
      if constexpr ((OCT & (OCT - 1)) == 0) {
#pragma unroll
        for (int d = OCT; d < 64; d *= 2) l = fminf(l, __shfl_xor(l, d)), u = fmaxf(u, __shfl_xor(u, d));
      } else {
#pragma unroll
        for (int q = 1; q < TOKENS; ++q) {
          l = fminf(l, __shfl(box.low[j], oct + q * OCT));
          u = fmaxf(u, __shfl(box.high[j], oct + q * OCT));
        }
      }
      lo[j >> 1] |= (__float_as_uint(l) >> 16) << (16 * (j & 1));  // exact: two significant bits
      hi[j >> 1] |= (__float_as_uint(u) >> 16) << (16 * (j & 1));
    }
    if (lane < OCT) {
      uint16_t *to = a.boxes[blockIdx.z] + (((int64_t)page * a.kv_heads + h) * 2) * D + oct * 8;
      *reinterpret_cast<u32x4 *>(to) = lo;
      *reinterpret_cast<u32x4 *>(to + D) = hi;
    }
  }

  wave_fence();
  store();
  for (int i0 = in_place + AHEAD; i0 < kept; i0 += AHEAD) {
    wave_fence();
    load(i0);
    wave_fence();
    store();
  }
}

// Tokens times heads from which on a lane has four tokens (8 heads of 128, us, a token a lane and four: runs of 64, 1024 tokens 4.8 and
// 4.4, 2048 7.0 and 5.0, 16 384 37 and 17; from everywhere 1024 4.8 and 8.0, 2048 7.6 and 9.5, 16 384 38 and 39).
constexpr int READ_RUNS = 16384;

// Eight channels of a held token's keys and values.
template <int D, int DT>
__device__ inline void read_token(const char *at, int place, int oct, u32x4 &k, u32x4 &v) {
  const int group = oct >> 2, lane = ((place >> 2) & 3) * 16, word = (place >> 4) * 4 + (place & 3);
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

// D / 8 lanes have a token and head, eight channels each.  301 tokens of 8 heads of 64: 3.6 us, the launch and two trips.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a) {
  constexpr int OCT = D / 8;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, rest = i / OCT;
  const int oct = i % OCT, h = rest % (uint32_t)a.kv_heads;
  const int64_t t = rest / (uint32_t)a.kv_heads;
  if (t >= a.tokens) return;
  const int64_t slot = a.slots[t];
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (slot >= 0 && slot < a.n_slots)
    read_token<D, DT>(a.pages + (slot / KV_PAGE * a.kv_heads + h) * (int64_t)kv_head_bytes(D), (int)(slot % KV_PAGE), oct, k, v);
  *reinterpret_cast<u32x4 *>(a.k + t * a.k_token + h * a.k_head + oct * 8) = k;
  *reinterpret_cast<u32x4 *>(a.v + t * a.v_token + h * a.v_head + oct * 8) = v;
}

// Four tokens a lane.  A page has four tokens' values of a channel beside each other, so four that follow each other, from a multiple
// of four on, take the loads of one; the fours of a workgroup's 64 tokens begin where its first token says.  Bound by memory: 30 011
// tokens of 8 heads of 128, 34 MB read (pages that come twice once) and 123 written, 36 us (4.3 TB/s); a token a lane 65.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_read_run_kernel(KvReadArgs a, int heads_at_once) {
  constexpr int OCT = D / 8, TILE = 64;
  const int64_t begin = (int64_t)blockIdx.x * TILE, end = min(begin + TILE, a.tokens);
  const int h0 = blockIdx.y * heads_at_once, heads = min(heads_at_once, a.kv_heads - h0);
  const int64_t ahead = a.slots[begin];
  const int shift = ahead >= 0 && begin + 1 < end && a.slots[begin + 1] == ahead + 1 ? (int)(ahead & 3) : 0;
  for (int i = threadIdx.x; i < (TILE / 4 + (shift != 0)) * heads * OCT; i += 256) {
    const int oct = i % OCT, rest = i / OCT, h = h0 + rest % heads, group = oct >> 2;
    const int64_t t0 = begin - shift + rest / heads * 4;
    if (t0 >= end) continue;
    int64_t slot[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) slot[j] = t0 + j >= begin && t0 + j < end ? a.slots[t0 + j] : -1;
    uint16_t *to_k = a.k + t0 * a.k_token + h * a.k_head + oct * 8, *to_v = a.v + t0 * a.v_token + h * a.v_head + oct * 8;
    if (slot[0] >= 0 && (slot[0] & 3) == 0 && slot[0] < a.n_slots && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 && slot[3] == slot[0] + 3) {
      const int place = (int)(slot[0] % KV_PAGE), lane = ((place >> 2) & 3) * 16, word = (place >> 4) * 4;
      const char *at = a.pages + (slot[0] / KV_PAGE * a.kv_heads + h) * (int64_t)kv_head_bytes(D);
      uint32_t kc[4], kb[4], w[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kc[j] = *reinterpret_cast<const uint32_t *>(at + (place + j) * (D / 2) + oct * 4);
        kb[j] = *reinterpret_cast<const uint8_t *>(at + kv_kscale_at(D) + (((place & 15) + j) * (D / 32) + group) * 4 + (place >> 4));
      }
      const uint32_t vb = *reinterpret_cast<const uint32_t *>(at + kv_vscale_at(D) + group * 64 + lane + word);
      const char *vp = at + kv_v_at(D) + group * 1024 + (lane + (oct & 1) * 8) * 16 + word;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const uint32_t *>(vp + j * 16) >> (2 * (oct & 2));  // the lane's half of each byte, lowest
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t vc = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) vc |= (w[c] >> (8 * j) & 15u) << (4 * c);
        const u32x4 k = kb[j] == 255 ? u32x4{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu} : held_row<DT>(kc[j], kb[j]);
        *reinterpret_cast<u32x4 *>(to_k + j * a.k_token) = k;
        *reinterpret_cast<u32x4 *>(to_v + j * a.v_token) = held_row<DT>(vc, vb >> (8 * j) & 0xff);
      }
    } else {
      // (all four tokens' loads before the first store; a token that is not there reads the cache's first)
      u32x4 k[4], v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool inside = slot[j] >= 0 && slot[j] < a.n_slots;
        const int64_t from = inside ? slot[j] : 0;
        read_token<D, DT>(a.pages + (from / KV_PAGE * a.kv_heads + h) * (int64_t)kv_head_bytes(D), (int)(from % KV_PAGE), oct, k[j], v[j]);
        if (!inside) k[j] = v[j] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (t0 + j < begin || t0 + j >= end) continue;
        *reinterpret_cast<u32x4 *>(to_k + j * a.k_token) = k[j];
        *reinterpret_cast<u32x4 *>(to_v + j * a.v_token) = v[j];
      }
    }
  }
}

template <int D, int DT>
int read_typed(const KvReadArgs &a, hipStream_t s) {
  const int64_t groups = (a.tokens * a.kv_heads * (D / 8) + 255) / 256;
  if (a.tokens * a.kv_heads >= READ_RUNS) {
    // the heads of a token beside each other, so that stores are long, but workgroups enough
    const int64_t tiles = (a.tokens + 63) / 64;
    int heads = a.kv_heads;
    while (heads > 1 && tiles * ((a.kv_heads + heads - 1) / heads) < 2048) heads = (heads + 1) / 2;
    hipLaunchKernelGGL((kv_read_run_kernel<D, DT>), dim3((unsigned)tiles, (unsigned)((a.kv_heads + heads - 1) / heads)), dim3(256), 0, s, a, heads);
  } else {
    hipLaunchKernelGGL((kv_read_kernel<D, DT>), dim3((unsigned)groups), dim3(256), 0, s, a);
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

template <int D>
int read_of(const KvReadArgs &a, int dtype, hipStream_t s) {
  return dtype == IVFPQ_KV_BF16 ? read_typed<D, IVFPQ_KV_BF16>(a, s) : read_typed<D, IVFPQ_KV_FP16>(a, s);
}

template <int D>
void move_of(const KvKeepArgs &a, int ring, hipStream_t s) {
  const dim3 grid((unsigned)(a.requests > 0 ? a.requests : 1), (unsigned)((a.kv_heads + 3) / 4), (unsigned)(a.n_caches + ring));
  if (a.max_nodes <= 64) hipLaunchKernelGGL((kv_move_kernel<D, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_move_kernel<D, false>), grid, dim3(256), 0, s, a);
}

}  // namespace

int launch_kv_move(const KvKeepArgs &a, int D, bool ring, hipStream_t s) {
  switch (D) {
    case 64: move_of<64>(a, ring, s); break;
    case 96: move_of<96>(a, ring, s); break;
    case 128: move_of<128>(a, ring, s); break;
    default: move_of<256>(a, ring, s); break;
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

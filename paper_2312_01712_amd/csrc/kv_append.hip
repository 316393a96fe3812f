// New keys and values into the pages of the 4-bit cache, and the boxes of their pages.
//
// The tokens of one page form a run of the list: slots that ascend by one and do not cross a
// page.  One workgroup has one run of one head, so nobody else touches the page's box or shares a
// byte: the box needs no atomics and does not depend on any order.  A lane has eight channels of four
// consecutive tokens (16-byte loads); four lanes share a scale.  Bound by memory: 4 D bytes read
// and 68 D / 64 written per token and head, plus 4 D if the rounded rows are wanted: 12 750 tokens of 8 heads of
// 128, 119 MB, in 31 us (3.8 TB/s); 48 tokens in 5.7 us.  Sizes are compared as bits and rows are rounded as they lie, two
// values an instruction: unpacked to 32 bits first it took 18 vector instructions an element and 34 us.

#include "kv_internal.h"

namespace ivfpq {

namespace {

// over the four lanes that share 32 channels (they are aligned to four)
__device__ inline uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));
}

// the value of the lane two further within its four
__device__ inline uint32_t quad_across(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Bits of the largest size among eight values: sizes order like their bits, infinities and NaN come last.
__device__ inline uint32_t largest(u32x4 raw) {
  u16x2 m = __builtin_bit_cast(u16x2, raw[0] & 0x7fff7fffu);
#pragma unroll
  for (int j = 1; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, raw[j] & 0x7fff7fffu));
  return max((uint32_t)m[0], (uint32_t)m[1]);
}

// The scale byte of 32 channels whose largest size has these bits.
template <int DT>
__device__ inline uint32_t scale_of(uint32_t top) {
  const int e = (int)(__float_as_uint(KvType<DT>::to_float((uint16_t)top)) >> 23) - 2;
  return (uint32_t)(e < 1 ? 1 : e > 254 ? 254 : e);
}

// eight values as codes, the first channel lowest
template <int DT>
__device__ inline uint32_t round_row(u32x4 raw, uint32_t b) {
  const float scale = __uint_as_float(b << 23);
  uint32_t w = 0;
  w = KvType<DT>::template round<0>(w, raw[0], scale);
  w = KvType<DT>::template round<1>(w, raw[1], scale);
  w = KvType<DT>::template round<2>(w, raw[2], scale);
  w = KvType<DT>::template round<3>(w, raw[3], scale);
  return w;
}

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

// four nibbles to the low halves of four bytes
__device__ inline uint32_t spread(uint32_t x) {
  x = (x | (x << 8)) & 0x00ff00ffu;
  return (x | (x << 4)) & 0x0f0f0f0fu;
}

// A run's tokens whose places p have (p / STEP) % of == turn: codes, scales, rounded rows; the lane's eight channels' box.
template <int D, int DT>
__device__ inline void write_run(const KvAppendArgs &a, int64_t i, int64_t slot0, int n, int h, int lane, int turn, int of,
                                 float *low, float *high) {
  constexpr int OCT = D / 8;          // lanes of a token
  constexpr int QUADS = 64 / OCT;     // groups of four tokens at a time
  constexpr int STEP = 4 * QUADS;
  const int place0 = (int)(slot0 % KV_PAGE);
  const int quad = lane / OCT, oct = lane % OCT;
  const bool active = lane < QUADS * OCT;
  const int group = oct >> 2;  // of 32 channels
  const uint64_t token_mask = (OCT == 64 ? ~0ull : ((1ull << OCT) - 1)) << (active ? quad * OCT : 0);
  const int64_t page = slot0 / KV_PAGE;
  char *at = a.pages + (page * a.kv_heads + h) * (int64_t)kv_head_bytes(D);
  const uint16_t *kp = a.k + h * a.k_head + oct * 8, *vp = a.v + h * a.v_head + oct * 8;

#pragma unroll
  for (int j = 0; j < 8; ++j) low[j] = __builtin_inff(), high[j] = -__builtin_inff();

  // groups of four places, from the one that holds the first token
  for (int g0 = (place0 & ~3) + turn * STEP; g0 < place0 + n; g0 += of * STEP) {
    const int t0 = g0 + quad * 4;  // place of the lane's first token
    const int64_t row0 = i + t0 - place0;
    const uint16_t *kr0 = kp + row0 * a.k_token, *vr0 = vp + row0 * a.v_token;
    u32x4 kr[4], vr[4];
    bool in[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int place = t0 + j;
      in[j] = active && place >= place0 && place < place0 + n;
      kr[j] = u32x4{0, 0, 0, 0};
      vr[j] = u32x4{0, 0, 0, 0};
      if (in[j]) {
        kr[j] = *reinterpret_cast<const u32x4 *>(kr0 + j * a.k_token);
        vr[j] = *reinterpret_cast<const u32x4 *>(vr0 + j * a.v_token);
      }
    }
    uint32_t kc[4], vc[4], ks[4], vs[4];
    bool bad[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t kt = largest(kr[j]), vt = largest(vr[j]);
      const uint64_t hit = __ballot(max(kt, vt) >= KvType<DT>::not_finite_bits);
      bad[j] = (hit & token_mask) != 0;
      if (hit != 0) {  // a token of this wavefront; zeros in the place of its values
        if (bad[j]) {
          kr[j] = vr[j] = u32x4{0, 0, 0, 0};
          kt = vt = 0;
        }
      }
      ks[j] = scale_of<DT>(quad_max(kt));
      vs[j] = scale_of<DT>(quad_max(vt));
      kc[j] = round_row<DT>(kr[j], ks[j]);
      vc[j] = round_row<DT>(vr[j], vs[j]);
    }
    const int64_t out0 = (row0 * a.kv_heads + h) * D + oct * 8, out_step = (int64_t)a.kv_heads * D;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (in[j]) {
        const int place = t0 + j;
        const u32x4 kh = held_row<DT>(kc[j], ks[j]);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float x = KvType<DT>::to_float((uint16_t)(kh[c >> 1] >> (16 * (c & 1))));
          low[c] = fminf(low[c], x);
          high[c] = fmaxf(high[c], x);
        }
        *reinterpret_cast<uint32_t *>(at + place * (D / 2) + oct * 4) = kc[j];
        if ((oct & 3) == 0)
          at[kv_kscale_at(D) + ((place % 16) * (D / 32) + group) * 4 + place / 16] = (char)(bad[j] ? 255 : ks[j]);
        if (a.k_rounded) {
          const u32x4 nan = u32x4{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
          *reinterpret_cast<u32x4 *>(a.k_rounded + out0 + j * out_step) = bad[j] ? nan : kh;
        }
        if (a.v_rounded) *reinterpret_cast<u32x4 *>(a.v_rounded + out0 + j * out_step) = held_row<DT>(vc[j], vs[j]);
      }
    // values: a byte has channels c and c + 16 of one token; the lane two further has the other
    // nibbles, and each of the two writes four of the eight bytes: channels 0-3 of the octet the
    // lower lane, 4-7 the upper one
    const bool upper = (oct & 2) != 0;  // this lane's channels are the high nibbles
    uint32_t bytes[4];                  // a token's four bytes
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t other = quad_across(vc[j]);
      const uint32_t lo = upper ? other >> 16 : vc[j] & 0xffff, hi = upper ? vc[j] >> 16 : other & 0xffff;
      bytes[j] = spread(lo) | (spread(hi) << 4);
    }
    if (in[0] || in[1] || in[2] || in[3]) {
      char *base = at + kv_v_at(D) + group * 1024 + ((t0 / 4) % 4) * 256 + (t0 / 16) * 4 + ((oct & 1) * 8 + (upper ? 4 : 0)) * 16;
      char *scales = at + kv_vscale_at(D) + group * 64 + ((t0 / 4) % 4) * 16 + (t0 / 16) * 4;
      if (in[0] && in[1] && in[2] && in[3]) {
        // four tokens' bytes of a channel together
        const uint32_t a01 = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x05010400), b01 = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x07030602);
        const uint32_t a23 = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x05010400), b23 = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x07030602);
        *reinterpret_cast<uint32_t *>(base) = __builtin_amdgcn_perm(a23, a01, 0x05040100);
        *reinterpret_cast<uint32_t *>(base + 16) = __builtin_amdgcn_perm(a23, a01, 0x07060302);
        *reinterpret_cast<uint32_t *>(base + 32) = __builtin_amdgcn_perm(b23, b01, 0x05040100);
        *reinterpret_cast<uint32_t *>(base + 48) = __builtin_amdgcn_perm(b23, b01, 0x07060302);
        if ((oct & 3) == 0) *reinterpret_cast<uint32_t *>(scales) = vs[0] | (vs[1] << 8) | (vs[2] << 16) | (vs[3] << 24);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (in[j]) {
#pragma unroll
            for (int c = 0; c < 4; ++c) base[c * 16 + j] = (char)(bytes[j] >> (8 * c));
            if ((oct & 3) == 0) scales[j] = (char)vs[j];
          }
      }
    }
  }
}

// The lanes' boxes of a run, and of `waves` wavefronts, joined with what the page's earlier tokens left.
template <int D>
__device__ inline void write_box(const KvAppendArgs &a, int64_t slot0, int h, int lane, int waves, float (*box)[2][8][64]) {
  constexpr int OCT = D / 8, QUADS = 64 / OCT;
  if (lane >= OCT) return;
  uint16_t *to = a.boxes + ((slot0 / KV_PAGE * a.kv_heads + h) * 2) * (int64_t)D + lane * 8;
  const bool begun = slot0 % KV_PAGE != 0;
  u32x4 old[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
  if (begun) {
    old[0] = *reinterpret_cast<const u32x4 *>(to);
    old[1] = *reinterpret_cast<const u32x4 *>(to + D);
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x = side ? -__builtin_inff() : __builtin_inff();
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int q = 0; q < QUADS; ++q) {
          const float y = box[w][side][j][lane + q * OCT];
          x = side ? fmaxf(x, y) : fminf(x, y);
        }
      if (begun) {
        const float was = __uint_as_float((old[side][j >> 1] >> (16 * (j & 1))) << 16);
        x = side ? fmaxf(x, was) : fminf(x, was);
      }
      const uint32_t half = __float_as_uint(x) >> 16;  // exact: two significant bits
      r[j >> 1] = (j & 1) ? r[j >> 1] | (half << 16) : half;
    }
    *reinterpret_cast<u32x4 *>(to + side * D) = r;
  }
}

// A workgroup has the runs that begin among `tile` tokens of the list, one head.  Long runs are written by its
// four wavefronts together, all of a page's loads in flight at once; short ones by a wavefront each.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a, int tile) {
  __shared__ float box[4][2][8][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y;
  const int64_t i0 = (int64_t)blockIdx.x * tile;
  // the slots of the tile's tokens and of the 63 behind the last, in one trip; all wavefronts look
  const int64_t none = -2;
  const int64_t here = i0 + lane < a.tokens ? a.slots[i0 + lane] : none;
  const int64_t there = lane < tile && i0 + 64 + lane < a.tokens ? a.slots[i0 + 64 + lane] : none;
  const int64_t ahead = i0 > 0 ? a.slots[i0 - 1] : none;
  int64_t prev = __shfl_up(here, 1);
  if (lane == 0) prev = ahead;
  // tokens that are the first of their run
  uint64_t heads = __ballot(lane < tile && here >= 0 && here < a.n_slots && (here % KV_PAGE == 0 || prev != here - 1));
  float low[8], high[8];
  auto keep = [&](int w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) box[w][0][j][lane] = low[j], box[w][1][j][lane] = high[j];
  };
  for (int run = 0; heads != 0; ++run, heads &= heads - 1) {
    const int first = __builtin_ctzll(heads);
    const int64_t i = i0 + first, slot0 = __shfl(here, first);
    // its length: a lane looks at each further place of the page
    const int64_t near = __shfl(here, (first + lane) & 63), far = __shfl(there, (first + lane) & 63);
    const bool on = lane < KV_PAGE - (int)(slot0 % KV_PAGE) && (first + lane < 64 ? near : far) == slot0 + lane;
    const uint64_t miss = ~__ballot(on);
    const int n = miss ? __builtin_ctzll(miss) : 64;
    if (n > 16) {
      write_run<D, DT>(a, i, slot0, n, h, lane, wave, 4, low, high);
      keep(wave);
      __syncthreads();
      if (wave == 0) write_box<D>(a, slot0, h, lane, 4, box);
      __syncthreads();
    } else if ((run & 3) == wave) {
      write_run<D, DT>(a, i, slot0, n, h, lane, 0, 1, low, high);
      keep(wave);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      write_box<D>(a, slot0, h, lane, 1, box + wave);
      __builtin_amdgcn_wave_barrier();
    }
  }
}

}  // namespace

template <int D>
static void append_of(const KvAppendArgs &a, int dtype, hipStream_t s) {
  // few tokens: a wavefront for each, should they be runs of one (48 tokens: 5.6 us, 16 a workgroup 14.9); many: most are not
  // the first of their run, or there are workgroups enough (2000 of one prompt: 8.2 us, 4 a workgroup 17.2; 3000 runs
  // of one: 41 and 43)
  const int tile = a.tokens <= 512 ? 4 : 16;
  const dim3 grid((unsigned)((a.tokens + tile - 1) / tile), (unsigned)a.kv_heads);
  if (dtype == IVFPQ_KV_BF16) hipLaunchKernelGGL((kv_append_kernel<D, IVFPQ_KV_BF16>), grid, dim3(256), 0, s, a, tile);
  else hipLaunchKernelGGL((kv_append_kernel<D, IVFPQ_KV_FP16>), grid, dim3(256), 0, s, a, tile);
}

int launch_kv_append(const KvAppendArgs &a, int D, int dtype, hipStream_t s) {
  switch (D) {
    case 64: append_of<64>(a, dtype, s); break;
    case 96: append_of<96>(a, dtype, s); break;
    case 128: append_of<128>(a, dtype, s); break;
    default: append_of<256>(a, dtype, s); break;
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

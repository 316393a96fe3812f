// Attention of drafted tokens over the paged 4-bit cache: what is held before them, and of themselves what their masks say.
//
// The kernels of kv_attention_kernels.h with masks, and one of its own for trees of some tokens: two to four tiles of 16 rows for a kv
// head are too many for the kernel of decoding, which unpacks a page for every tile, and too few for that of chunks, which unpacks
// pages into LDS for many.  Here a wavefront has pages of its own, as in decoding, but every fragment that it unpacks feeds the
// products of two tiles, and two wavefronts read a page at the same time for two tiles each.  Pages come into LDS without passing
// registers, so that three wavefronts fit a SIMD.

#include "kv_attention_kernels.h"

namespace ivfpq {

namespace {

constexpr int NT = 4;  // tiles of 16 rows of a unit, two of a wavefront

// Half a page (keys or values, with their scales) into LDS.  All lanes take part in every load, as a branch of some of them around
// one may not be joined with another's: the lanes behind the scales' end read their last bytes again, and the place has room for them.
template <int D>
constexpr int half_loads() { return D / 32 + (2 * D + 255) / 256; }
template <int D>
constexpr int half_bytes() { return 32 * D + (2 * D + 255) / 256 * 256; }

template <int D>
__device__ inline void fetch_half(const char *from, char *to, int lane) {
  typedef __attribute__((address_space(1))) void *global;
  typedef __attribute__((address_space(3))) void *local;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) __builtin_amdgcn_global_load_lds((global)(from + i * 1024 + lane * 16), (local)(to + i * 1024), 16, 0, 0);
#pragma unroll
  for (int i = 0; i < 2 * D; i += 256)
    __builtin_amdgcn_global_load_lds((global)(from + 32 * D + min(i + lane * 4, 2 * D - 4)), (local)(to + 32 * D + i), 4, 0, 0);
}

// Loads into LDS are counted with those into registers, in order: all but the youngest N are done.
template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Nothing is still to be read from LDS.
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The rows of a unit in LDS; 16 bytes more than a query takes, so that rows begin in different banks.
template <int D>
struct RowsInLds {
  uint16_t query[16 * NT][D + 8];
  int32_t token[16 * NT], low[16 * NT];
};

// All rows of the unit's tiles, those behind its last as that one: what is done with them is not kept, but their masks are looked at.
template <int D>
__device__ inline void place_rows(const KvAttnArgs &a, const Unit &u, int rows, RowsInLds<D> &to, int tid) {
  const int placed = (rows + 15) / 16 * 16;
  const uint32_t flip = a.negative ? 0x80008000u : 0u;  // a negative scale: of the rows' values
  for (int job = tid; job < placed * (D / 8); job += 256) {
    const int row = job / (D / 8), part = job % (D / 8), i = u.tile * (16 * NT) + min(row, rows - 1);
    const int64_t t = u.t0 + i / a.group;
    u32x4 x = *reinterpret_cast<const u32x4 *>(a.q + t * a.q_token + (u.head * a.group + i % a.group) * a.q_head + part * 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] ^= flip;
    *reinterpret_cast<u32x4 *>(&to.query[row][part * 8]) = x;
    if (part == 0) {
      to.token[row] = (int32_t)t;
      const int here = a.window > 0 ? min(max(a.tree_positions[t], u.pos0), u.pos0 + u.fresh - 1) : 0;
      to.low[row] = a.window > 0 ? max(here - a.window, -1) : -1;
    }
  }
}

// Byte I of w where the conversions look for a scale's exponent; they look at nothing else of it (compared for every exponent with
// the other bits clear and set).
template <int I>
__device__ inline float scale_byte(uint32_t w) { return __uint_as_float(I == 3 ? w >> 1 : w << (23 - 8 * I)); }

// Scales of four tokens, where the conversions look for them.
__device__ inline void four_scales(uint32_t sc, float *f) {
  f[0] = scale_byte<0>(sc);
  f[1] = scale_byte<1>(sc);
  f[2] = scale_byte<2>(sc);
  f[3] = scale_byte<3>(sc);
}

// As unpack_tokens.
template <int DT>
__device__ inline void four_tokens(uint32_t w, const float *f, u32x4 &lo, u32x4 &hi, int half) {
  const uint32_t a = KvType<DT>::template unpack<0>(w, f[0]), b = KvType<DT>::template unpack<1>(w, f[1]);
  const uint32_t c = KvType<DT>::template unpack<2>(w, f[2]), d = KvType<DT>::template unpack<3>(w, f[3]);
  lo[half * 2] = __builtin_amdgcn_perm(b, a, 0x05040100);
  hi[half * 2] = __builtin_amdgcn_perm(b, a, 0x07060302);
  lo[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x05040100);
  hi[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

// Which channels a lane has as a row of the values' products.  A page's scales are of 32 channels, two channels c and c + 16 lie in a byte.
// With the channels of an accumulator one block's (as they lie) a lane meets all blocks and unpacks a scale for every byte.  So a
// row has C = D / 32 bytes next to each other, all of one block: 16 scales of a page instead of 16 C, 48 of 420 vector instructions
// less for 128 channels.  The order of a row's bytes is another for each two rows (for 128), so that sixteen lanes, and eight, read from
// different banks.  Three blocks do not go into 16 rows evenly: 96 channels are taken as they lie.
template <int D>
constexpr bool ONE_BLOCK = D != 96;

// byte v of row m, of the 16 C of a token
template <int D>
__device__ inline int pair_of(int m, int v) {
  constexpr int C = D / 32;
  if constexpr (!ONE_BLOCK<D>) return v * 16 + m;
  const int x = m * C / 8;
  return m * C + (v ^ (x & (C - 1)) ^ x / C);
}

// The pages of a unit that a wavefront takes: [at, end), every `step`-th.
struct Walk {
  const int32_t *table;
  int at, end, step, numbers, lo, any_low;
  uint64_t todo;

  __device__ inline void look(const KvAttnArgs &a, const Unit &u, int lane) {  // 64 entries at a time, a lane each
    const int k = at + step * lane, c = lo + k;
    numbers = k < end && c < a.width && c * KV_PAGE < u.kv && c * KV_PAGE + KV_PAGE - 1 > any_low ? table[c] : -1;
    todo = __ballot((uint32_t)numbers < (uint64_t)a.n_pages);
  }
  __device__ inline int next(const KvAttnArgs &a, const Unit &u, int lane, int &first) {
    while (!todo) {
      at += step * 64;
      if (at >= end) return -1;
      look(a, u, lane);
    }
    const int j = __builtin_ctzll(todo);
    todo &= todo - 1;
    first = (lo + at + step * j) * KV_PAGE;
    return __builtin_amdgcn_readlane(numbers, j);
  }
};

// A unit's rows, N tiles of 16 from `tile` on, over the wavefront's pages, the first of which is on its way.  Keys and values of a
// page have a place each in LDS, of the wavefront alone; the next page's are requested as soon as these are used.
template <int D, int DT, int N>
__device__ inline void tiles_pages(const KvAttnArgs &a, const Unit &u, Walk &walk, int page, int first, int lane, const RowsInLds<D> &in,
                                   int tile, char *keys, Row<D> *r) {
  constexpr int C = D / 32, LOADS = half_loads<D>();
  constexpr float SLACK = 8.0f, LIFT = DT == IVFPQ_KV_FP16 ? 15.0f - SLACK : 0.0f;
  const char *heads = a.pages + u.head * (int64_t)kv_head_bytes(D);
  const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
  const int past = min(u.pos0, u.kv);
  // what no row sees more than (as positions do not follow the order of tokens)
  const int clear_low = a.window > 0 ? u.pos0 + u.fresh - 1 - a.window : -1;
  char *values = keys + half_bytes<D>();
  int turn = blockIdx.x / 256 % 3;
  const uint16_t(*query)[D + 8] = in.query + tile * 16;
  const int32_t *token = in.token + tile * 16, *low = in.low + tile * 16;

  while (page >= 0) {
    int first_next = 0;
    const int page_next = walk.next(a, u, lane, first_next);
    wait_loads<LOADS>();  // the keys are there
    // The oldest wavefront of a SIMD goes first where priorities are equal: it would end early and leave the others alone.  So each has the
    // highest priority for every third page (16 tokens behind 300 001: wavefronts live 91 % of the kernel's time instead of 79 %).
    switch (turn) {
      case 0: __builtin_amdgcn_s_setprio(0); turn = 1; break;
      case 1: __builtin_amdgcn_s_setprio(1); turn = 2; break;
      default: __builtin_amdgcn_s_setprio(2); turn = 0; break;
    }
    const bool masked = first + KV_PAGE > past || first <= clear_low;
    u32x4 pf[N][2];
    asm volatile("" : "+v"(lane));  // (so that the places below are computed here and not kept: registers are short)
    const int row = lane & 15, g = lane >> 4;
    const int at = pair_of<D>(row, 0) / 16 * 1024 + g * 256 + pair_of<D>(row, 0) % 16 * 16;
    auto bytes = [&](int v) { return *reinterpret_cast<const u32x4 *>(values + (ONE_BLOCK<D> ? at ^ v * 16 : v * 1024 + lane * 16)); };
    auto scales_of = [&](int v) { return *reinterpret_cast<const u32x4 *>(values + 32 * D + (ONE_BLOCK<D> ? at / 16 & ~15 : v * 64 + g * 16)); };
    {
      f32x4 s[N][4];
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) s[k][tt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      const uint32_t *scales = reinterpret_cast<const uint32_t *>(keys + kv_kscale_at(D)) + row * C;
      const uint32_t ks0 = scales[(C * g) / 4], ks1 = C == 3 || C == 8 ? scales[(C * g + C - 1) / 4] : ks0;
      const char *codes = keys + row * (D / 2) + g * (D / 8);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        u32x4 q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = *reinterpret_cast<const u32x4 *>(&query[k * 16 + row][g * (D / 4) + c * 8]);
        auto tile = [&](auto TT) {
          constexpr int tt = decltype(TT)::value;
          const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + tt * 8 * D + c * 4);
          const float s0 = scale_byte<tt>(ks0), s1 = C == 3 || C == 8 ? scale_byte<tt>(ks1) : s0;
          const float sc = C == 8 ? (c < 4 ? s0 : s1) : C == 3 ? ((C * g + c) / 4 == (C * g) / 4 ? s0 : s1) : s0;
          u32x4 x;
          x[0] = KvType<DT>::template unpack<0>(w, sc);
          x[1] = KvType<DT>::template unpack<1>(w, sc);
          x[2] = KvType<DT>::template unpack<2>(w, sc);
          x[3] = KvType<DT>::template unpack<3>(w, sc);
#pragma unroll
          for (int k = 0; k < N; ++k) s[k][tt] = KvType<DT>::mfma(x, q[k], s[k][tt]);
        };
        tile(std::integral_constant<int, 0>());
        tile(std::integral_constant<int, 1>());
        tile(std::integral_constant<int, 2>());
        tile(std::integral_constant<int, 3>());
      }
      wait_lds();
      if (page_next >= 0) fetch_half<D>(heads + page_next * page_bytes, keys, lane);
      if (masked) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const uint64_t sees = tree_sees(a, u, token[k * 16 + row], low[k * 16 + row], first) >> (4 * g);
          const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
          for (int e = 0; e < 16; ++e) s[k][e >> 2][e & 3] = half[e >> 3] >> (16 * (e >> 2 & 1) + (e & 3)) & 1 ? s[k][e >> 2][e & 3] : -__builtin_inff();
        }
      }
      // as page_maximum, the tiles beside each other
      float top[N];
      bool grows = false;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        top[k] = s[k][0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top[k] = fmaxf(top[k], s[k][e >> 2][e & 3]);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        top[k] = row_max(top[k]) * a.scale2 - LIFT;
        grows = grows || top[k] > r[k].m + SLACK;
      }
      if (__any(grows)) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float m = top[k] > r[k].m + SLACK ? top[k] : r[k].m, f = m > r[k].m ? __builtin_amdgcn_exp2f(r[k].m - m) : 1.0f;
          r[k].l *= f;
#pragma unroll
          for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) r[k].o[ct][i] *= f;
          r[k].m = m;
        }
      }
      // the values are there: only the next page's keys were requested after them
      if (page_next >= 0) wait_loads<LOADS>();
      else wait_loads<0>();
      if (u.kv - first < KV_PAGE) {  // what no token of the request's wrote must not meet a weight of 0 as an infinity
        if (lane < 4 * C) {
          u32x4 *at = reinterpret_cast<u32x4 *>(values + 32 * D + lane * 16);
          u32x4 x = *at;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int m = min(max(u.kv - first - (16 * d + 4 * (lane & 3)), 0), 4);
            const uint32_t keep = m >= 4 ? 0xffffffffu : (1u << (8 * m)) - 1u;
            x[d] = (x[d] & keep) | (0x01010101u & ~keep);
          }
          *at = x;
        }
        wait_lds();
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        page_weights<D, DT>(s[k], r[k], pf[k], a.scale2);
      }
    }
    float f[16];  // scales of the lane's 16 tokens
#pragma unroll
    for (int v = 0; v < C; ++v) {
      const u32x4 w = bytes(v);
      if (v == 0 || !ONE_BLOCK<D>) {
        const u32x4 sc = scales_of(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) four_scales(sc[i], f + 4 * i);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 lo, hi;
#pragma unroll
        for (int half = 0; half < 2; ++half) four_tokens<DT>(w[h * 2 + half], f + h * 8 + half * 4, lo, hi, half);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          r[k].o[2 * v] = KvType<DT>::mfma(lo, pf[k][h], r[k].o[2 * v]);
          r[k].o[2 * v + 1] = KvType<DT>::mfma(hi, pf[k][h], r[k].o[2 * v + 1]);
        }
      }
    }
    wait_lds();
    if (page_next >= 0) fetch_half<D>(heads + page_next * page_bytes + 34 * D, values, lane);
    page = page_next;
    first = first_next;
  }
}

// Units of up to NT tiles, shared out among workgroups as in kv_rows16_kernel; a workgroup's wavefronts have two tiles each and take the
// unit's pages in turn, two for each pair of tiles or four for the only one, and add up through LDS.  Bound by the issue of
// instructions (vector units 64 % busy, matrix units 28 %): a page and two tiles are 390 instructions of the vector units, half
// of them unpacking, and 64 products.  16 tokens of 32 heads behind 300 001, 79 GFLOP, 328 MB, 114 us and 9 of joining (16 rows a tile as in
// decoding: 168 in all; units of two tiles, which read every page twice, 118 and 10); trees of up to 32 tokens, 64 heads, behind 24
// contexts to 33 000, 117 GFLOP, 184 us with joining (in the kernel of chunks 245, in units of two tiles 188).  Three tiles a wavefront with two
// wavefronts a SIMD took 160 and 282 us, four, which leave a few values to memory in the loop, 169 and 328; eight wavefronts a
// workgroup 75 us where four took 60 (one request of 100 000).  Scaled products of the 4-bit codes themselves would save unpacking keys, but sum to
// 2^-17 of the sizes' sum only, and take no 16-bit queries.
template <int D, int DT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D <= 128 ? 3 : 2))) void kv_tiles_kernel(KvAttnArgs a) {
  constexpr int TR = 16 * NT;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float *buf = reinterpret_cast<float *>(lds);  // [4][16][D + 4], where the pages are before
  auto &in = *reinterpret_cast<RowsInLds<D> *>(lds + 8 * half_bytes<D>());
  float(*ml)[16][2] = reinterpret_cast<float(*)[16][2]>(&in + 1);  // [4]
  int *sums = reinterpret_cast<int *>(ml + 4);                    // [4]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4;
  // Shares that follow each other on one of the chip's eight parts, which have an L2 each: the tiles of a request and head read the same
  // pages at the same time.
  const int wg = gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;

  Requests q = {a.prefix, nullptr, nullptr, nullptr};
  int total;
  if (a.scanned) {
    total = uniform(a.prefix[a.requests]);
  } else {
    q.prefix = sums + 4;                                            // [requests], and [requests + 1] each:
    q.t0 = q.prefix + a.requests;
    q.kv = q.t0 + a.requests + 1;
    q.pos0 = q.kv + a.requests + 1;
    total = scan_units<TR, 256, true>(a, q, sums, tid);
  }
  const Share share = share_of(a, total, wg);
  if (tid == 0 && !a.whole && share.begin >= share.end) a.borders[(int64_t)wg * BORDER_INTS] = 0;
  for (int at = share.begin; at < share.end;) {
    int offset;
    Unit u = unit_at<TR, false, true>(a, q, at, offset);
    const int rows = min(TR, u.fresh * a.group - u.tile * TR), tiles = (rows + 15) / 16, weight = unit_weight(rows);
    // indexes of the unit: what it counts beside its pages, then these
    const int extra = a.whole ? 0 : UNIT_EXTRA, entries = a.whole ? u.pages : weight * (u.pages + extra);
    const int taken = a.whole ? entries : min(entries - offset, share.end - at);
    const int first = a.whole ? 0 : max(offset / weight - extra, 0), end = a.whole ? u.pages : max((offset + taken) / weight - extra, 0);
    // up to two tiles: four wavefronts with a page each; more: two for each two tiles, so that a page is read at about the same
    // time by both and comes from memory once
    const int own = weight == 2 ? wave >> 1 : 0;
    Walk walk = {a.table + (int64_t)u.req * a.width, first + (weight == 2 ? wave & 1 : wave), end, 4 / weight, -1, u.lo,
                 a.window > 0 ? u.pos0 - a.window : -1, 0};
    if (walk.at < walk.end) walk.look(a, u, lane);
    int position = 0;
    const int page = walk.next(a, u, lane, position);
    char *place = lds + wave * (2 * half_bytes<D>());
    if (page >= 0) {
      const char *from = a.pages + u.head * (int64_t)kv_head_bytes(D) + page * (a.kv_heads * (int64_t)kv_head_bytes(D));
      fetch_half<D>(from, place, lane);
      fetch_half<D>(from + 34 * D, place + half_bytes<D>(), lane);
    }
    place_rows<D>(a, u, rows, in, tid);
    Row<D> r[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      r[k].m = -__builtin_inff();
      r[k].l = 0.0f;
#pragma unroll
      for (int ct = 0; ct < D / 16; ++ct) r[k].o[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __syncthreads();
    if (tiles - 2 * own == 1) tiles_pages<D, DT, 1>(a, u, walk, page, position, lane, in, 2 * own, place, r);
    else tiles_pages<D, DT, 2>(a, u, walk, page, position, lane, in, 2 * own, place, r);
    const int64_t slot = 2 * (int64_t)wg + (at != share.begin);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (k < tiles) {
        r[k].l = row_sum(r[k].l);
        __syncthreads();  // the pages are used, or the buffer is free again
        if (g == 0) ml[wave][lane & 15][0] = r[k].m, ml[wave][lane & 15][1] = r[k].l;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct)
          if constexpr (ONE_BLOCK<D>) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int p = pair_of<D>(g * 4 + i, ct / 2);
              buf[(wave * 16 + (lane & 15)) * (D + 4) + p / 16 * 32 + p % 16 + ct % 2 * 16] = r[k].o[ct][i];
            }
          } else {
            *reinterpret_cast<f32x4 *>(buf + (wave * 16 + (lane & 15)) * (D + 4) + ct * 16 + g * 4) = r[k].o[ct];
          }
        __syncthreads();
        if (weight == 1) {
          join_waves<D, DT, NT>(a, u, rows, taken == entries, slot, ml, buf, tid, k);
        } else {
          join_waves<D, DT, NT, 2>(a, u, rows, taken == entries, slot, ml, buf, tid, k);
          if (2 + k < tiles) join_waves<D, DT, NT, 2>(a, u, rows, taken == entries, slot, ml + 2, buf + 2 * 16 * (D + 4), tid, 2 + k);
        }
      }
    __syncthreads();
    const int next = at + (a.whole ? 1 : taken);
    u.pages = entries;
    if (tid == 0 && !a.whole && next == share.end) leave_border(a, share, u, wg, at, rows);
    at = next;
  }
  clear_rest<D, 256>(a, wg, gridDim.x, tid);
}

// How a call is cut.  tiles: by kv_tiles_kernel.
struct TreeShape : Shape {
  bool tiles;
  int64_t units;
};

TreeShape tree_shape(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_nodes, int window, int64_t width) {
  TreeShape s;
  const int64_t nodes = max_nodes < tokens ? max_nodes : tokens, rows = nodes * group;  // rows of a request and head, at most
  int64_t most = width;  // pages of a unit
  if (window > 0 && ((int64_t)window + nodes) / KV_PAGE + 2 < most) most = ((int64_t)window + nodes) / KV_PAGE + 2;
  // 8 kv heads of 128, us.  16 rows and fewer: the kernel of decoding.  Little work (pages that tiles of 16 rows read): that one up to
  // 64 rows, as its first page takes fewer trips and more workgroups share it (32 rows: 32 requests of 4000 49, here 55; 64 rows: one of
  // 8000 21 and 30, 32 of 1500 44 and 50), this one beyond if there is next to none (128 rows: one of 500 20 in the kernel of chunks and
  // here 19, of 8000 34 and 35).  Otherwise this one up to 96 rows (32: 16 of 16 000 97 and 79; 64: the same 169 and 118, 16 of 8000 92 and
  // 72; 96: 32 of 4000 110 and 89), the kernels of chunks beyond (128: 32 of 1500 50 and 64, of 4000 119 and 121; 256: 157 and 209), but where
  // requests have fewer tokens than the largest, whose tiles they leave part empty (64 of up to 8000, trees of up to 128 rows 147
  // and 101, 512 365 and 286).  `work` counts the table's width, as the host does not know what requests hold; each of its borders
  // rests on two or three shapes, which differ by little there.
  const int64_t work = ((tokens * group + 15) / 16 + requests) * kv_heads * most;
  const bool ragged = tokens * 8 <= requests * nodes * 7 && rows <= 512;
  if (rows <= 64) s.tiles = rows > 16 && work >= 49152;
  else s.tiles = ragged || (work < 49152 ? work < 8192 : rows <= 96);
  if (!s.tiles) {
    static_cast<Shape &>(s) = shape_of(tokens, requests, kv_heads, group, D, max_nodes, window, 0, width);
    return s;
  }
  const bool narrow = most <= WHOLE_PAGES;
  s.tile_rows = 16 * NT;
  const int64_t units = s.units = (tokens * group / s.tile_rows + requests) * kv_heads;
  const int fill = D <= 128 ? 768 : 256;
  const int64_t surely = window > 0 ? (window + tokens) / KV_PAGE + 2 : width;
  s.whole = narrow || units * 2 * ((surely < width ? surely : width) + UNIT_EXTRA) > 0x7fffffff;
  const int shares = units * most / 2 >= fill ? fill : (int)(units * most / 2 + 1);
  s.n_wg = s.whole ? (int)units : shares;
  if (s.n_wg < 1) s.n_wg = 1;
  s.prefix = up256((size_t)(requests + 1) * 4);
  s.borders = narrow ? 0 : up256((size_t)shares * BORDER_INTS * 4);
  s.ml = narrow ? 0 : up256((size_t)shares * 2 * s.tile_rows * 2 * 4);
  s.o = narrow ? 0 : up256((size_t)shares * 2 * s.tile_rows * D * 4);
  return s;
}

template <int D, int DT>
int tiles_of(KvAttnArgs a, const TreeShape &sh, hipStream_t s) {
  // Lists of the requests in LDS, or from a launch before: also where the lists would leave room for two workgroups instead of three (160 KB in
  // steps of 1280 bytes; 34 requests of 8 tokens of 64 heads of 128 behind 3000: 85 us with the lists, 70 with the launch; 28: 59 and 63).
  const size_t own = 8 * (size_t)half_bytes<D>() + sizeof(RowsInLds<D>) + 4 * 16 * 2 * 4 + 4 * 4;
  const size_t all = ((size_t)a.requests + 3 * (size_t)(a.requests + 1)) * 4;
  auto three = [](size_t bytes) { return 3 * ((bytes + 1279) / 1280) <= 128; };
  a.scanned = a.requests > SCAN_REQUESTS || (three(own) && !three(own + all));
  if (a.scanned) {
    hipLaunchKernelGGL(kv_scan_kernel, dim3(1), dim3(1024), 0, s, a, sh.tile_rows, 1);
    KV_HIP_TRY(hipGetLastError());
  }
  const size_t lds = own + (a.scanned ? 0 : all);
  int rc;
  if ((rc = allow_lds(&kv_tiles_kernel<D, DT>, lds))) return rc;
  hipLaunchKernelGGL((kv_tiles_kernel<D, DT>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
  KV_HIP_TRY(hipGetLastError());
  if (a.whole || a.n_wg == 1) return IVFPQ_OK;
  const int64_t most = a.tokens * (int64_t)a.group;
  const int rows = (int)(most < sh.tile_rows ? most : sh.tile_rows);
  // few units of dozens of parts each: a workgroup a row of a unit (of a share, most of which leave no unit across their border:
  // 14 us for 8 units of 64 rows, now 9); many of two or three: a workgroup 256 / (D / 4) rows (800 units over 768 shares: 21 us and 7)
  if (sh.n_wg >= 8 * sh.units) {
    hipLaunchKernelGGL((kv_join_kernel<D, DT, true>), dim3((unsigned)sh.units, (unsigned)rows), dim3(256), 0, s, a, sh.tile_rows, a.n_wg - 1);
  } else {
    constexpr int SETS = 256 / (D / 4);
    hipLaunchKernelGGL((kv_join_kernel<D, DT, false>), dim3((unsigned)(a.n_wg - 1), (unsigned)((rows + SETS - 1) / SETS)), dim3(256), 0, s, a,
                       sh.tile_rows, 0);
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

template <int D, int DT>
int tree_attention_of(const KvAttnArgs &a, const TreeShape &sh, hipStream_t s) {
  if (!sh.tiles) return attention_of<D, DT, true>(a, sh, s);
  return tiles_of<D, DT>(a, sh, s);
}

template <int D>
int tree_attention_typed(const KvAttnArgs &a, int dtype, const TreeShape &sh, hipStream_t s) {
  return dtype == IVFPQ_KV_BF16 ? tree_attention_of<D, IVFPQ_KV_BF16>(a, sh, s) : tree_attention_of<D, IVFPQ_KV_FP16>(a, sh, s);
}

}  // namespace

size_t kv_tree_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_nodes, int window,
                                   int64_t width) {
  const TreeShape s = tree_shape(tokens, requests, kv_heads, group, D, max_nodes, window, width);
  return s.prefix + s.borders + s.ml + s.o;
}

int launch_kv_tree_attention(const KvAttnArgs &args, int D, int dtype, int max_nodes, char *workspace, hipStream_t s) {
  KvAttnArgs a = args;
  const TreeShape sh = tree_shape(a.tokens, a.requests, a.kv_heads, a.group, D, max_nodes, a.window, a.width);
  if (!launch_fits(sh.n_wg, sh.tile_rows == 256 || (sh.tile_rows == 128 && D == 256) ? 512 : 256)) {
    set_error("kv_tree_attention: %d workgroups are too many for one launch", sh.n_wg);
    return IVFPQ_ERR_UNSUPPORTED;
  }
  place_workspace(a, sh, workspace);
  switch (D) {
    case 64: return tree_attention_typed<64>(a, dtype, sh, s);
    case 96: return tree_attention_typed<96>(a, dtype, sh, s);
    case 128: return tree_attention_typed<128>(a, dtype, sh, s);
    default: return tree_attention_typed<256>(a, dtype, sh, s);
  }
}

}  // namespace ivfpq

// Attention of a step's new tokens over the paged 4-bit cache, all pages or selected ones, or with masks: what the units that launch
// it share (kv_attention.hip, kv_tree_attention.hip).
//
// The running form of the softmax: with s_j = scale log2(e) q . k_j, a row keeps m = max s_j (or a number near it),
// l = sum 2^(s_j - m) and o = sum 2^(s_j - m) v_j and multiplies l and o by 2^(m_old - m_new) when m
// grows; parts of the keys joined the same way.  Sums and statistics are in 32 bits.  Weights are
// rounded to the cache's type for the second product, whose other factor, a held value, is exact in it: half a unit of the
// result's type at most, as rounding the result, and the products run at the 16-bit rate.
//
// Layout.  A wavefront works on S^T = K Q^T and O^T = V^T P^T, 16 rows (query heads of one kv head, tokens above
// them) at a time, so that a lane holds one row's statistics and the exponentials of the first
// product are, in place, the second operand of the second: lane (g, row) has keys 16 tt + 4 g + i, and
// the page stores the values in this order of tokens.
//
// Two kernels here; trees have a third (kv_tree_attention.hip).  kv_rows16_kernel: 16 rows or fewer share a page (decode, selected
// pages); its wavefronts have pages of their own, held in registers from memory to the products.  kv_rows_kernel: many rows share a
// page (chunks of prompts); a workgroup unpacks a page into LDS once and its wavefronts have 32 rows each.

#pragma once

#include <type_traits>

#include "kv_internal.h"

namespace ivfpq {

namespace {

constexpr int SCAN_REQUESTS = 512;  // more than these: their units are scanned by a launch of its own
constexpr int UNIT_EXTRA = 8;       // pages that a unit in tiles counts beside its own: see unit_weight
constexpr int WHOLE_PAGES = 32;     // tables up to this width: a workgroup has whole units, nothing is joined

// over the four lanes that hold a row: lanes 16 apart
__device__ inline float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float row_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// values that are the same in all lanes, in scalar registers
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// pages [lo, lo + n) that any new token of a request sees; n >= 1
struct Range {
  int lo, n;
};

__device__ inline Range request_pages(int kv, int fresh, int window, int width) {
  Range g = {0, 1};
  const int past = max(kv - fresh, 0);
  if (window > 0 && past - window + 1 > 0) g.lo = (past - window + 1) / KV_PAGE;
  g.lo = min(g.lo, width - 1);
  g.n = max(min((int)(((int64_t)kv + KV_PAGE - 1) / KV_PAGE), width) - g.lo, 1);
  return g;
}

// What a wavefront reads of a page and head.
template <int D>
struct Page {
  uint32_t k[4][D / 32], ks[2];
  u32x4 v[D / 32], vs[D / 32];

  __device__ inline void load(const char *at, int lane) {
    const int row = lane & 15, g = lane >> 4;
    constexpr int C = D / 32;  // dwords of keys a lane has of a token: channels [g D/4, (g + 1) D/4)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const uint32_t *p = reinterpret_cast<const uint32_t *>(at + (tt * 16 + row) * (D / 2) + g * (D / 8));
      if constexpr (C == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
        for (int j = 0; j < 4; ++j) k[tt][j] = x[j];
      } else if constexpr (C == 8) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(p), y = *reinterpret_cast<const u32x4 *>(p + 4);
        for (int j = 0; j < 4; ++j) k[tt][j] = x[j], k[tt][4 + j] = y[j];
      } else if constexpr (C == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
        k[tt][0] = x[0], k[tt][1] = x[1];
      } else {
        struct three { uint32_t x[3]; };
        const three x = *reinterpret_cast<const three *>(p);
        for (int j = 0; j < 3; ++j) k[tt][j] = x.x[j];
      }
    }
    const uint32_t *s = reinterpret_cast<const uint32_t *>(at + kv_kscale_at(D)) + row * C;
    ks[0] = s[(C * g) / 4];
    ks[1] = s[(C * g + C - 1) / 4];
    const char *vp = at + kv_v_at(D) + lane * 16, *vsp = at + kv_vscale_at(D) + g * 16;
#pragma unroll
    for (int p = 0; p < C; ++p) {
      v[p] = *reinterpret_cast<const u32x4 *>(vp + p * 1024);
      vs[p] = *reinterpret_cast<const u32x4 *>(vsp + p * 64);
    }
  }

  // Values behind the request's last token were never written in this request's time: whatever
  // is there must not meet a weight of 0 as an infinity.  held: tokens of this page.
  __device__ inline void cut(int held, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int d = 0; d < 4; ++d) {  // dword d: tokens 16 d + 4 g + i, byte i
      const int n = min(max(held - (16 * d + 4 * g), 0), 4);
      const uint32_t keep = n >= 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
#pragma unroll
      for (int p = 0; p < D / 32; ++p) vs[p][d] = (vs[p][d] & keep) | (0x01010101u & ~keep);
    }
  }
};

// A row's state: a lane has (m, l) of row lane % 16 (l: of its own keys) and the channels
// 16 ct + 4 (lane / 16) + i of its output.
template <int D>
struct Row {
  float m, l;
  f32x4 o[D / 16];
};

template <int D, int DT>
__device__ inline void page_scores(const Page<D> &pg, const u32x4 *qf, int lane, f32x4 *s) {
  constexpr int C = D / 32;
  const int g = lane >> 4;
  auto tile = [&](auto TT) {
    constexpr int tt = decltype(TT)::value;
    const float s0 = kv_scale<tt>(pg.ks[0]), s1 = C == 3 || C == 8 ? kv_scale<tt>(pg.ks[1]) : s0;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float sc = C == 8 ? (c < 4 ? s0 : s1) : C == 3 ? ((C * g + c) / 4 == (C * g) / 4 ? s0 : s1) : s0;
      u32x4 a;
      a[0] = KvType<DT>::template unpack<0>(pg.k[tt][c], sc);
      a[1] = KvType<DT>::template unpack<1>(pg.k[tt][c], sc);
      a[2] = KvType<DT>::template unpack<2>(pg.k[tt][c], sc);
      a[3] = KvType<DT>::template unpack<3>(pg.k[tt][c], sc);
      acc = KvType<DT>::mfma(a, qf[c], acc);
    }
    s[tt] = acc;
  };
  tile(std::integral_constant<int, 0>());
  tile(std::integral_constant<int, 1>());
  tile(std::integral_constant<int, 2>());
  tile(std::integral_constant<int, 3>());
}

template <int DT, int I>
__device__ inline uint32_t unpack_v(uint32_t w, uint32_t scales) {
  return KvType<DT>::template unpack<I>(w, kv_scale<I>(scales));
}

// Four tokens of channels c (low nibbles, to lo) and c + 16 (to hi).
template <int DT>
__device__ inline void unpack_tokens(uint32_t w, uint32_t sc, u32x4 &lo, u32x4 &hi, int half) {
  const uint32_t a = unpack_v<DT, 0>(w, sc), b = unpack_v<DT, 1>(w, sc), c = unpack_v<DT, 2>(w, sc), d = unpack_v<DT, 3>(w, sc);
  lo[half * 2] = __builtin_amdgcn_perm(b, a, 0x05040100);
  hi[half * 2] = __builtin_amdgcn_perm(b, a, 0x07060302);
  lo[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x05040100);
  hi[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

template <int D, int DT>
__device__ inline void page_values(const Page<D> &pg, const u32x4 *pf, f32x4 *o) {
#pragma unroll
  for (int p = 0; p < D / 32; ++p)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 lo, hi;
#pragma unroll
      for (int half = 0; half < 2; ++half) unpack_tokens<DT>(pg.v[p][u * 2 + half], pg.vs[p][u * 2 + half], lo, hi, half);
      o[2 * p] = KvType<DT>::mfma(lo, pf[u], o[2 * p]);
      o[2 * p + 1] = KvType<DT>::mfma(hi, pf[u], o[2 * p + 1]);
    }
}

// The largest product of a page joins a row's maximum; what the row has so far shrinks with it.  first: position of the
// page's first key; the row sees (low, high], low >= -1.  Products are compared unscaled (scale2 > 0): one multiply-add an
// exponential.  slack: a maximum that grows by less (in powers of two) is left, and weights go up to 2^slack.  That
// costs accuracy: without it the largest weight is a power of two, which its rounding leaves alone.  Chunks take it (8: 333 us
// for 348, the results 0.0023 off for 0.0019 in bf16), decoding, which waits for memory, does not.
// In fp16, whose smallest step is 2^-24, m is the maximum less 15 - slack: weights go up to 2^15, and one loses 2^-40 of the
// largest (with a slack 2^-32) to that step instead of 2^-25, which many small ones together would miss.  l and o carry
// the same factor, so that nothing else knows of it.
// With a tree `sees` has a bit for each key of the page instead.
template <int D, int DT, bool TREE = false>
__device__ inline void page_maximum(f32x4 *s, Row<D> &r, int g, float scale2, bool masked, int first, int low, int high,
                                    float slack, uint64_t sees = 0) {
  if (TREE && masked) {
    sees >>= 4 * g;
    const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[tt][i] = half[tt >> 1] >> (16 * (tt & 1) + i) & 1 ? s[tt][i] : -__builtin_inff();
  } else if (masked) {
    const int from = low - first - g * 4, to = high - first - g * 4;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[tt][i] = tt * 16 + i > from && tt * 16 + i <= to ? s[tt][i] : -__builtin_inff();
  }
  float top = s[0][0];
#pragma unroll
  for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e >> 2][e & 3]);
  const float lift = DT == IVFPQ_KV_FP16 ? 15.0f - slack : 0.0f;
  top = row_max(top) * scale2 - lift;
  if (__any(top > r.m + slack)) {
    const float m = fmaxf(r.m, top), f = m > r.m ? __builtin_amdgcn_exp2f(r.m - m) : 1.0f;
    r.l *= f;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) r.o[ct][i] *= f;
    r.m = m;
  }
}

// Products into weights, as the second operand of V^T P^T, and their sum.
template <int D, int DT>
__device__ inline void page_weights(const f32x4 *s, Row<D> &r, u32x4 *pf, float scale2) {
  const float base = r.m == -__builtin_inff() ? 0.0f : r.m;  // a row that saw nothing so far: every weight is 0
#pragma unroll
  for (int tt = 0; tt < 4; ++tt) {
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i], scale2, -base));
    r.l += (e[0] + e[1]) + (e[2] + e[3]);
    pf[tt >> 1][(tt & 1) * 2] = KvType<DT>::pack(e[0], e[1]);
    pf[tt >> 1][(tt & 1) * 2 + 1] = KvType<DT>::pack(e[2], e[3]);
  }
}

// One page into 16 rows.
template <int D, int DT, bool TREE = false>
__device__ inline void page_step(const Page<D> &pg, const u32x4 *qf, Row<D> &r, int lane, float scale2, bool masked,
                                 int first, int low, int high, uint64_t sees = 0) {
  f32x4 s[4];
  u32x4 pf[2];
  page_scores<D, DT>(pg, qf, lane, s);
  page_maximum<D, DT, TREE>(s, r, lane >> 4, scale2, masked, first, low, high, 0.0f, sees);
  page_weights<D, DT>(s, r, pf, scale2);
  page_values<D, DT>(pg, pf, r.o);
}

template <int DT>
__device__ inline void store_row(uint16_t *to, const float *x, int n) {
  for (int c = 0; c < n; c += 2) *reinterpret_cast<uint32_t *>(to + c) = KvType<DT>::pack(x[c], x[c + 1]);
}

// Rows of a unit: row i of tile `tile` (TR rows each) of a group is token i / G, head i % G (of the kv head); a group
// is a request or, with selected pages, a token.
struct Unit {
  int head, tile, lo, pages;         // kv head, tile, first page (or 0: entries of a list), pages
  int t0, fresh, kv, req, pos0;      // first token, tokens, held, request (-1: none), position of the first token
  int first;                         // index of its first page among all units' pages
};

// What the workgroups know of each request: units before it and what it takes to place its rows.
struct Requests {
  int32_t *prefix;            // [requests]
  int32_t *t0, *kv, *pos0;    // in LDS, or null: read from the step's arrays
};

// Units of up to 64 rows in tiles (TILES): what an index counts.  With up to 32 rows a workgroup's four wavefronts take four pages at a time,
// with more, two: a page counts for as much time.  Beside its pages a unit counts about as many as finding, placing and joining
// it takes (in units of 32 rows, 24 trees of up to 32 tokens, 64 heads, behind up to 33 000: 247 us without, 215 with 6, 220 with 12).
__device__ inline int unit_weight(int rows) { return rows > 32 ? 2 : 1; }

struct TileUnits {
  int tiles, full, last, head;  // units of a head, indexes of a unit of 64 rows, of the last one, of a head
};
__device__ inline TileUnits tile_units(int64_t rows, int pages, bool whole) {
  TileUnits t;
  t.tiles = (int)((rows + 63) / 64);
  t.full = whole ? 1 : 2 * (pages + UNIT_EXTRA);
  t.last = whole ? 1 : unit_weight((int)(rows - 64 * (int64_t)(t.tiles - 1))) * (pages + UNIT_EXTRA);
  t.head = (t.tiles - 1) * t.full + t.last;
  return t;
}

// Whole units are counted instead of their pages.  The host sees to it that all of them stay below 2^31.
template <int TR, bool TILES>
__device__ inline int units_of(const KvAttnArgs &a, int fresh, int kv) {
  if (fresh <= 0) return 0;
  if constexpr (TILES) return a.kv_heads * tile_units((int64_t)fresh * a.group, request_pages(kv, fresh, a.window, a.width).n, a.whole).head;
  const int n = (int)(((int64_t)fresh * a.group + TR - 1) / TR) * a.kv_heads;
  return a.whole ? n : n * request_pages(kv, fresh, a.window, a.width).n;
}

// Position of a request's first new token.  Where the table's width has cut the request its length does not say.
__device__ inline int first_position(const KvAttnArgs &a, int t0, int fresh, int kv) {
  if (kv < a.width * KV_PAGE) return kv - fresh;
  return fresh > 0 ? a.positions[t0] : 0;
}

// Units before every request, by the whole workgroup; returns their sum.
template <int TR, int THREADS, bool TILES = false>
__device__ inline int scan_units(const KvAttnArgs &a, const Requests &q, int *sums, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  int carry = 0;
  for (int b = 0; b < a.requests; b += THREADS) {
    const int r = b + tid;
    int n = 0;
    if (r < a.requests) {
      const int t0 = a.q_start[r], fresh = min(a.q_start[r + 1], a.tokens) - t0, kv = a.kv_lens[r];
      n = units_of<TR, TILES>(a, fresh, kv);
      if (q.t0) {
        q.t0[r] = t0;
        q.kv[r] = kv;
        q.pos0[r] = first_position(a, t0, fresh, kv);
        if (r == a.requests - 1) q.t0[r + 1] = t0 + fresh;
      }
    }
    int x = lanes_up_to(n);
    if (b > 0) __syncthreads();
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += sums[w];
    if (r < a.requests) q.prefix[r] = carry + x - n;
    for (int w = 0; w < THREADS / 64; ++w) carry += sums[w];
  }
  __syncthreads();
  return uniform(carry);
}

__global__ __launch_bounds__(1024) void kv_scan_kernel(KvAttnArgs a, int tile_rows, int tiles) {
  __shared__ int sums[16];
  const Requests q = {a.prefix, nullptr, nullptr, nullptr};
  const int total = tiles ? scan_units<64, 1024, true>(a, q, sums, threadIdx.x)
                      : tile_rows == 16 ? scan_units<16, 1024>(a, q, sums, threadIdx.x)
                      : tile_rows == 64 ? scan_units<64, 1024>(a, q, sums, threadIdx.x)
                      : tile_rows == 128 ? scan_units<128, 1024>(a, q, sums, threadIdx.x)
                                         : scan_units<256, 1024>(a, q, sums, threadIdx.x);
  if (threadIdx.x == 0) a.prefix[a.requests] = total;
}

// The unit that index `at` belongs to, and which of its pages that is.
template <int TR, bool SEL, bool TILES = false>
__device__ inline Unit unit_at(const KvAttnArgs &a, const Requests &q, int at, int &offset) {
  Unit u;
  int k;  // unit of its group
  if constexpr (SEL) {
    const int tiles = (a.group + TR - 1) / TR, n = a.whole ? 1 : a.n_select, per = a.kv_heads * tiles;
    k = at / n;
    offset = at % n;
    u.t0 = k / per;
    k %= per;
    u.head = k / tiles, u.tile = k % tiles;
    u.lo = 0, u.pages = a.n_select, u.fresh = 1;
    const int r = uniform(a.token_req[u.t0]);
    u.pos0 = uniform(a.positions[u.t0]);
    u.req = (uint32_t)r < (uint32_t)a.requests ? r : -1;
    u.kv = u.req >= 0 ? uniform(a.kv_lens[u.req]) : 0;
  } else {
    int lo = 0, hi = a.requests;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (uniform(q.prefix[mid]) <= at) lo = mid;
      else hi = mid;
    }
    u.req = lo;
    if (q.t0) {
      u.t0 = uniform(q.t0[lo]);
      u.fresh = uniform(q.t0[lo + 1]) - u.t0;
      u.kv = uniform(q.kv[lo]);
      u.pos0 = uniform(q.pos0[lo]);
    } else {
      u.t0 = uniform(a.q_start[lo]);
      u.fresh = min(uniform(a.q_start[lo + 1]), a.tokens) - u.t0;
      u.kv = uniform(a.kv_lens[lo]);
      u.pos0 = uniform(first_position(a, u.t0, u.fresh, u.kv));
    }
    const Range pr = request_pages(u.kv, u.fresh, a.window, a.width);
    const int rest = at - uniform(q.prefix[lo]);
    if constexpr (TILES) {
      const TileUnits t = tile_units((int64_t)u.fresh * a.group, pr.n, a.whole);
      u.head = rest / t.head;
      u.tile = min(rest % t.head / t.full, t.tiles - 1);
      offset = rest % t.head - u.tile * t.full;
    } else {
      const int tiles = (int)(((int64_t)u.fresh * a.group + TR - 1) / TR), n = a.whole ? 1 : pr.n;
      k = rest / n;
      offset = rest % n;
      u.head = k / tiles, u.tile = k % tiles;
    }
    u.lo = pr.lo, u.pages = pr.n;
  }
  u.first = at - offset;
  return u;
}

// A workgroup's share: [begin, end) of all units' pages, or whole units.
struct Share {
  int span, begin, end;
};

__device__ inline Share share_of(const KvAttnArgs &a, int total, int wg) {
  Share s;
  s.span = a.whole ? 1 : max((int)(((int64_t)total + a.n_wg - 1) / a.n_wg), 4);
  const int64_t begin = (int64_t)wg * s.span;
  s.begin = (int)min(begin, (int64_t)total);
  s.end = (int)min(begin + s.span, (int64_t)total);
  return s;
}

// What a workgroup leaves about the unit that goes across the border behind its share, if it began in it:
// shares that have some of it (0: there is none), whether it is not the first unit in its first
// share, first token, tile, kv head, rows.
constexpr int BORDER_INTS = 8;

__device__ inline void leave_border(const KvAttnArgs &a, const Share &s, const Unit &u, int wg, int at, int rows) {
  const bool across = u.first + u.pages > s.end && u.first >= s.begin;
  int32_t *b = a.borders + (int64_t)wg * BORDER_INTS;
  b[0] = across ? (u.first + u.pages - 1) / s.span - wg + 1 : 0;
  b[1] = at != s.begin;
  b[2] = u.t0;
  b[3] = u.tile;
  b[4] = u.head;
  b[5] = rows;
}

// The row that a lane works on, and which keys the rows of its 16 see: the row itself (low, high]; every row those in
// (clear_low, clear_high]; none those outside (any_low, any_high].
struct Place {
  int64_t t;
  int hq, low, high, clear_low, clear_high, any_low, any_high;
};

template <int TR, bool TREE = false>
__device__ inline Place place_of(const KvAttnArgs &a, const Unit &u, int rows, int in_tile) {
  Place p;
  const int i = u.tile * TR + min(in_tile, rows - 1);
  p.t = u.t0 + i / a.group;
  p.hq = u.head * a.group + i % a.group;
  if constexpr (TREE) {
    // positions do not follow the order of tokens: what is clear is said for all of the request's
    p.high = u.kv - 1;
    p.low = a.window > 0 ? max(min(max(a.tree_positions[p.t], u.pos0), u.pos0 + u.fresh - 1) - a.window, -1) : -1;
    p.clear_high = min(u.pos0, u.kv) - 1;
    p.any_high = u.kv - 1;
    p.clear_low = a.window > 0 ? max(u.pos0 + u.fresh - 1 - a.window, -1) : -1;
    p.any_low = a.window > 0 ? max(u.pos0 - a.window, -1) : -1;
    return p;
  }
  // the lane's 16 rows are in order of tokens: their first and last decide
  const int i0 = u.tile * TR + min(in_tile & ~15, rows - 1), i1 = u.tile * TR + min(in_tile | 15, rows - 1);
  const int pos = u.pos0 + i / a.group, pos_a = u.pos0 + i0 / a.group, pos_b = u.pos0 + i1 / a.group;
  p.high = min(pos, u.kv - 1);
  p.low = a.window > 0 ? max(pos - a.window, -1) : -1;
  p.clear_high = uniform(min(pos_a, u.kv - 1));
  p.any_high = uniform(min(pos_b, u.kv - 1));
  p.clear_low = uniform(a.window > 0 ? max(pos_b - a.window, -1) : -1);
  p.any_low = uniform(a.window > 0 ? max(pos_a - a.window, -1) : -1);
  return p;
}

// Which keys of the page that begins at position `first` a tree's token sees, a bit each: those held before the new tokens and above
// `low`, and new ones by its mask.
__device__ inline uint64_t tree_sees(const KvAttnArgs &a, const Unit &u, int64_t t, int low, int first) {
  const int n = min(u.pos0, u.kv) - first;  // keys of the page before the new tokens
  uint64_t x = 0;
  if (n < 64) {
    const uint64_t *mask = a.masks + t * a.words;
    const int at = max(-n, 0) >> 6, shift = max(-n, 0) & 63;
    const uint64_t word = at < a.words ? mask[at] : 0;
    x = n > 0 ? word << n : word >> shift;
    if (shift != 0 && at + 1 < a.words) x |= mask[at + 1] << (64 - shift);
    const int rest = u.kv - first;  // keys that are held
    if (rest < 64) x &= rest > 0 ? (1ull << rest) - 1 : 0;
  }
  uint64_t held = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0;
  const int out = low + 1 - first;  // keys that the window leaves out
  if (out > 0) held &= out < 64 ? ~0ull << out : 0;
  return x | held;
}

// A lane's part of its row as the second operand of K Q^T: channels g D/4 + 8 c + 0 .. 7.
template <int D>
__device__ inline void load_row(const KvAttnArgs &a, int64_t t, int hq, int g, u32x4 *qf) {
  const uint16_t *at = a.q + t * a.q_token + hq * a.q_head + g * (D / 4);
  const uint32_t flip = a.negative ? 0x80008000u : 0u;  // a negative scale: of the row's values
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    qf[c] = *reinterpret_cast<const u32x4 *>(at + c * 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) qf[c][j] ^= flip;
  }
}

__device__ inline float lse_of(float m, float l) {
  return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// A unit's rows from the wavefronts that had some of its pages each: to the result, or to the workspace.
// tile: which 16 of a unit of NT tiles.
template <int D, int DT, int NT = 1, int WAVES = 4>
__device__ inline void join_waves(const KvAttnArgs &a, const Unit &u, int rows, bool whole, int64_t slot, float (*ml)[16][2],
                                  float *buf, int tid, int tile = 0) {
  // buf [WAVES][16][D + 4], ml [WAVES]
  const int row = tid >> 4, part = tid & 15;
  float m = -__builtin_inff(), l = 0.0f, f[WAVES];
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[w][row][0]);
  const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    f[w] = __builtin_amdgcn_exp2f(ml[w][row][0] - base);
    l += f[w] * ml[w][row][1];
  }
  float x[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    x[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x[c] += f[w] * buf[(w * 16 + row) * (D + 4) + part * (D / 16) + c];
  }
  if (whole) {
    if (tile * 16 + row < rows) {
      const int i = (u.tile * NT + tile) * 16 + row;
      const int64_t t = u.t0 + i / a.group;
      const int hq = u.head * a.group + i % a.group;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) x[c] *= inv;
      store_row<DT>(a.out + t * a.out_token + hq * a.out_head + part * (D / 16), x, D / 16);
      if (a.lse && part == 0) a.lse[t * (a.kv_heads * a.group) + hq] = lse_of(m, l);
    }
  } else {
    const int64_t at = (slot * NT + tile) * 16 + row;
    float *to = a.part_o + at * D + part * (D / 16);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) to[c] = x[c];
    if (part == 0) {
      a.part_ml[at * 2] = m;
      a.part_ml[at * 2 + 1] = l;
    }
  }
}

// rows that stand for no token: behind the last request's tokens
template <int D, int THREADS>
__device__ inline void clear_rest(const KvAttnArgs &a, int64_t wg, int64_t n_wg, int tid) {
  const int heads = a.kv_heads * a.group;
  int64_t t = a.requests > 0 ? a.q_start[a.requests] : 0;
  if (t < 0) t = 0;
  const int64_t n = (a.tokens - t) * heads;
  for (int64_t i = wg * THREADS + tid; i < n * (D / 8); i += n_wg * THREADS) {
    const int64_t row = i / (D / 8);
    *reinterpret_cast<u32x4 *>(a.out + (t + row / heads) * a.out_token + (row % heads) * a.out_head + (i % (D / 8)) * 8) =
        u32x4{0, 0, 0, 0};
    if (a.lse && i % (D / 8) == 0) a.lse[t * heads + row] = -__builtin_inff();
  }
}

// A workgroup has an equal share of all (request or token, head, tile, page) units, in this order: ragged
// requests cost no balance.  Its four wavefronts take the share's pages in turn, each with its own
// softmax state; what a workgroup has of a unit whose pages it does not have all goes to the
// workspace, and kv_join_kernel adds up.  Where the table is narrow a workgroup has a whole unit instead.
// Bound by reading the pages (decode: 16 rows or fewer share a page): one token of 520 001, 566 MB, 109 us (5.2 TB/s); 40
// requests of 700 to 33 000, 361 MB, 91 us; 24 x 64 selected pages, 108 MB, 29 us; 334 tokens of 12 heads of 64 6.2 us, the
// chain of its first trips to memory.
template <int D, int DT, bool SEL, bool TREE = false>
__global__ __launch_bounds__(256, 2) void kv_rows16_kernel(KvAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float *buf = reinterpret_cast<float *>(lds);                                     // [4][16][D + 4]
  float(*ml)[16][2] = reinterpret_cast<float(*)[16][2]>(buf + 4 * 16 * (D + 4));  // [4]
  int *sums = reinterpret_cast<int *>(ml + 4);                                    // [4]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4;
  const int wg = blockIdx.x;

  Requests q = {a.prefix, nullptr, nullptr, nullptr};
  int total;
  if constexpr (SEL) {
    total = a.tokens * a.kv_heads * ((a.group + 15) / 16) * (a.whole ? 1 : a.n_select);
  } else if (a.scanned) {
    total = uniform(a.prefix[a.requests]);
  } else {
    q.prefix = sums + 4;                                            // [requests], and [requests + 1] each:
    q.t0 = q.prefix + a.requests;
    q.kv = q.t0 + a.requests + 1;
    q.pos0 = q.kv + a.requests + 1;
    total = scan_units<16, 256>(a, q, sums, tid);
  }
  const Share share = share_of(a, total, wg);
  if (tid == 0 && !a.whole && share.begin >= share.end) a.borders[(int64_t)wg * BORDER_INTS] = 0;
  for (int at = share.begin; at < share.end;) {
    int offset;
    const Unit u = unit_at<16, SEL>(a, q, at, offset);
    const int n = a.whole ? u.pages : min(u.pages - offset, share.end - at);
    const int rows = min(16, u.fresh * a.group - u.tile * 16);
    const Place p = place_of<16, TREE>(a, u, rows, lane & 15);
    const int32_t *table = a.table + (int64_t)max(u.req, 0) * a.width;
    const int32_t *list = SEL ? a.selected + ((int64_t)u.t0 * a.kv_heads + u.head) * a.n_select : nullptr;
    const char *heads = a.pages + u.head * (int64_t)kv_head_bytes(D);
    const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
    u32x4 qf[D / 32];
    load_row<D>(a, p.t, p.hq, g, qf);
    Row<D> r;
    r.m = -__builtin_inff();
    r.l = 0.0f;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) r.o[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int k1 = offset + n;
    // the wavefront's entries offset + wave, + 4, ...: a lane looks 64 of them up at a time
    for (int k0 = offset + wave; k0 < k1; k0 += 4 * 64) {
      const int k = k0 + 4 * lane;
      int c = u.lo + k, page = -1;
      if constexpr (SEL) c = list[min(k, k1 - 1)];
      if (k < k1 && u.req >= 0) {
        // not a column that no row sees anything of, nor one without a page in the cache
        if ((uint32_t)c < (uint32_t)a.width && c * KV_PAGE <= p.any_high && c * KV_PAGE + KV_PAGE - 1 > p.any_low) page = table[c];
      }
      uint64_t todo = __ballot((uint32_t)page < (uint64_t)a.n_pages);
      auto fetch = [&](Page<D> &pg, uint64_t left) {
        pg.load(heads + __builtin_amdgcn_readlane(page, __builtin_ctzll(left)) * page_bytes, lane);
      };
      auto step = [&](Page<D> &pg, uint64_t left) {
        const int first = __builtin_amdgcn_readlane(c, __builtin_ctzll(left)) * KV_PAGE;
        if (first + KV_PAGE > u.kv) pg.cut(u.kv - first, lane);
        const bool masked = first + KV_PAGE - 1 > p.clear_high || first <= p.clear_low;
        const uint64_t sees = TREE && masked ? tree_sees(a, u, p.t, p.low, first) : 0;
        page_step<D, DT, TREE>(pg, qf, r, lane, a.scale2, masked, first, p.low, p.high, sees);
      };
      // a page is requested while the one before it is worked on (256 channels: no registers for two)
      if constexpr (D <= 128) {
        Page<D> even, odd;
        if (todo) fetch(even, todo);
        while (todo) {
          const uint64_t then = todo & (todo - 1);
          if (then) fetch(odd, then);
          step(even, todo);
          if (!then) break;
          todo = then & (then - 1);
          if (todo) fetch(even, todo);
          step(odd, then);
        }
      } else {
        for (; todo; todo &= todo - 1) {
          Page<D> pg;
          fetch(pg, todo);
          step(pg, todo);
        }
      }
    }
    r.l = row_sum(r.l);
    __syncthreads();  // the buffer is free again
    if (g == 0) ml[wave][lane & 15][0] = r.m, ml[wave][lane & 15][1] = r.l;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
      *reinterpret_cast<f32x4 *>(buf + (wave * 16 + (lane & 15)) * (D + 4) + ct * 16 + g * 4) = r.o[ct];
    __syncthreads();
    join_waves<D, DT>(a, u, rows, n == u.pages, 2 * (int64_t)wg + (at != share.begin), ml, buf, tid);
    const int next = at + (a.whole ? 1 : n);
    if (tid == 0 && !a.whole && next == share.end) leave_border(a, share, u, wg, at, rows);
    at = next;
  }
  if constexpr (!SEL) clear_rest<D, 256>(a, wg, gridDim.x, tid);  // (selected: rows without a request are units)
}

// Fragments of an unpacked page in LDS, 64 lanes of 16 bytes each, as the matrix units take them:
// keys (tt, c) at tt C + c, values (channel tile ct, token half u) at 4 C + 2 ct + u; C = D / 32.
template <int D>
constexpr int page_fragments() { return 4 * (D / 32) + 2 * (D / 16); }

// What a wavefront unpacks of a page: its share of the keys' and values' fragments, a job each of two (keys of 96
// channels: one) fragments.
template <int D, int DT, int WAVES>
struct Unpack {
  static constexpr int C = D / 32, KF = C % 2 ? 1 : 2, KJOBS = 4 * C / KF, VJOBS = 2 * C;
  static constexpr int KN = (KJOBS + WAVES - 1) / WAVES, VN = (VJOBS + WAVES - 1) / WAVES;
  uint32_t k[KN][KF], ks[KN];
  u32x2 v[VN], vs[VN];

  __device__ inline void load(const char *at, int wave, int lane) {
    const int row = lane & 15, g = lane >> 4;
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      const int job = n * WAVES + wave, tt = job / (C / KF), c = job % (C / KF) * KF;
      if (job < KJOBS) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(at + (tt * 16 + row) * (D / 2) + g * (D / 8)) + c;
        if constexpr (KF == 2) {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
          k[n][0] = x[0], k[n][1] = x[1];
        } else {
          k[n][0] = p[0];
        }
        // the scale of channels 8 (C g + c) ..: the fragments of a job are within 32 channels
        ks[n] = (uint32_t)*reinterpret_cast<const uint8_t *>(at + kv_kscale_at(D) + (row * C + (C * g + c) / 4) * 4 + tt);
      }
    }
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int job = n * WAVES + wave, p = job >> 1, u = job & 1;
      if (job < VJOBS) {
        v[n] = *reinterpret_cast<const u32x2 *>(at + kv_v_at(D) + p * 1024 + lane * 16 + u * 8);
        vs[n] = *reinterpret_cast<const u32x2 *>(at + kv_vscale_at(D) + p * 64 + g * 16 + u * 8);
      }
    }
  }

  // held: tokens of this page; what is behind them must not meet a weight of 0 as an infinity
  __device__ inline void store(u32x4 *to, int wave, int lane, int held) {
    const int g = lane >> 4;
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      const int job = n * WAVES + wave, tt = job / (C / KF), c = job % (C / KF) * KF;
      if (job < KJOBS) {
        const float sc = __uint_as_float(ks[n] << 23);
#pragma unroll
        for (int f = 0; f < KF; ++f) {
          u32x4 x;
          x[0] = KvType<DT>::template unpack<0>(k[n][f], sc);
          x[1] = KvType<DT>::template unpack<1>(k[n][f], sc);
          x[2] = KvType<DT>::template unpack<2>(k[n][f], sc);
          x[3] = KvType<DT>::template unpack<3>(k[n][f], sc);
          to[(tt * C + c + f) * 64 + lane] = x;
        }
      }
    }
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int job = n * WAVES + wave, p = job >> 1, u = job & 1;
      if (job < VJOBS) {
        u32x4 lo, hi;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t sc = vs[n][half];
          if (held < KV_PAGE) {
            const int m = min(max(held - (32 * u + 16 * half + 4 * g), 0), 4);
            const uint32_t keep = m >= 4 ? 0xffffffffu : (1u << (8 * m)) - 1u;
            sc = (sc & keep) | (0x01010101u & ~keep);
          }
          unpack_tokens<DT>(v[n][half], sc, lo, hi, half);
        }
        to[(4 * C + 4 * p + u) * 64 + lane] = lo;
        to[(4 * C + 4 * p + 2 + u) * 64 + lane] = hi;
      }
    }
  }
};

// A barrier that orders the workgroup's LDS accesses and leaves loads from memory on their way.
__device__ inline void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Many rows of one kv head: a workgroup unpacks a page into LDS, one ahead of the one worked on (two
// buffers, a barrier a page), and each of its wavefronts has NQ times 16 rows with their queries, weights
// and results in registers.  A fragment read from LDS feeds NQ products.  Bound by the matrix units (35 % busy)
// and the vector ones (50 %; an exponential takes 16 cycles): 2048 tokens of 32 heads behind 8190, 309 GFLOP, 333 us
// (929 TFLOP/s; an 8192^3 library product reaches 1203).
template <int D, int DT, int WAVES, int NQ, bool TREE = false>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, WAVES * NQ == 4 ? 3 : 2))) void kv_rows_kernel(KvAttnArgs a) {
  constexpr int TR = WAVES * NQ * 16, C = D / 32, FRAGS = page_fragments<D>(), THREADS = 64 * WAVES;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  u32x4 *frag = reinterpret_cast<u32x4 *>(lds);                              // [2][FRAGS][64]
  int *sums = reinterpret_cast<int *>(frag + 2 * FRAGS * 64);                // [WAVES]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4;
  const int wg = blockIdx.x;

  Requests q = {a.prefix, nullptr, nullptr, nullptr};
  int total;
  if (a.scanned) {
    total = uniform(a.prefix[a.requests]);
  } else {
    q.prefix = sums + WAVES;
    q.t0 = q.prefix + a.requests;
    q.kv = q.t0 + a.requests + 1;
    q.pos0 = q.kv + a.requests + 1;
    total = scan_units<TR, THREADS>(a, q, sums, tid);
  }
  const Share share = share_of(a, total, wg);
  if (tid == 0 && !a.whole && share.begin >= share.end) a.borders[(int64_t)wg * BORDER_INTS] = 0;
  for (int at = share.begin; at < share.end;) {
    int offset;
    const Unit u = unit_at<TR, false>(a, q, at, offset);
    const int n = a.whole ? u.pages : min(u.pages - offset, share.end - at);
    const int rows = min(TR, u.fresh * a.group - u.tile * TR);
    Place p[NQ];
    u32x4 qf[NQ][C];
    Row<D> r[NQ];
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      p[k] = place_of<TR, TREE>(a, u, rows, wave * (NQ * 16) + k * 16 + (lane & 15));
      load_row<D>(a, p[k].t, p[k].hq, g, qf[k]);
      r[k].m = -__builtin_inff();
      r[k].l = 0.0f;
#pragma unroll
      for (int ct = 0; ct < D / 16; ++ct) r[k].o[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // pages that some row of the tile sees
    const int last = u.tile * TR + rows - 1;
    const int see_high = TREE ? u.kv - 1 : min(u.pos0 + last / a.group, u.kv - 1);
    const int see_low = a.window > 0 ? u.pos0 + (TREE ? 0 : u.tile * TR / a.group) - a.window + 1 : 0;
    const int c0 = max(u.lo + offset, max(see_low, 0) / KV_PAGE), c1 = min(u.lo + offset + n, (see_high + KV_PAGE) / KV_PAGE);
    const int32_t *table = a.table + (int64_t)u.req * a.width;
    const char *heads = a.pages + u.head * (int64_t)kv_head_bytes(D);
    const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
    const bool idle = wave * (NQ * 16) >= rows;  // no row of this wavefront is one

    Unpack<D, DT, WAVES> job;
    // the columns with a page in the cache, in order: a lane looks one of 64 up at a time
    int block = c0, numbers = -1;
    uint64_t todo = 0;
    auto look = [&]() {
      numbers = block + lane < c1 ? table[block + lane] : -1;
      todo = __ballot((uint32_t)numbers < (uint64_t)a.n_pages);
    };
    auto next_page = [&](int &c) -> int {
      while (!todo) {
        block += 64;
        if (block >= c1) return -1;
        look();
      }
      const int j = __builtin_ctzll(todo);
      todo &= todo - 1;
      c = block + j;
      return __builtin_amdgcn_readlane(numbers, j);
    };
    look();
    // the page worked on is in LDS, the next in registers, requested a page's work ago
    int c = 0, page = next_page(c), cur = 0;
    int cn = 0, pn = -1;
    lds_barrier();  // the buffers are free again
    if (page >= 0) {
      job.load(heads + page * page_bytes, wave, lane);
      job.store(frag, wave, lane, u.kv - c * KV_PAGE);
      pn = next_page(cn);
      if (pn >= 0) job.load(heads + pn * page_bytes, wave, lane);
    }
    lds_barrier();
    while (page >= 0) {
      const u32x4 *fr = frag + cur * (FRAGS * 64) + lane;
      const int first = c * KV_PAGE;
      bool skip[NQ], all = true;
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        skip[k] = first > p[k].any_high || first + KV_PAGE - 1 <= p[k].any_low;
        all = all && skip[k];
      }
      if (!idle && !all) {
        // four fragments are on their way from LDS while the products of the four before them run
        u32x4 x[2][4];
        auto read = [&](int f, u32x4 *to) {
#pragma unroll
          for (int b = 0; b < 4; ++b) to[b] = fr[(f + b) * 64];
        };
        f32x4 s[NQ][4];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int k = 0; k < NQ; ++k) s[k][tt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        read(0, x[0]);
#pragma unroll
        for (int f = 0; f < 4 * C; f += 4) {
          if (f + 4 < 4 * C) read(f + 4, x[(f / 4 + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int k = 0; k < NQ; ++k) s[k][(f + b) / C] = KvType<DT>::mfma(x[(f / 4) & 1][b], qf[k][(f + b) % C], s[k][(f + b) / C]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
          const bool masked = first + KV_PAGE - 1 > p[k].clear_high || first <= p[k].clear_low;
          const uint64_t sees = TREE && masked ? tree_sees(a, u, p[k].t, p[k].low, first) : 0;
          page_maximum<D, DT, TREE>(s[k], r[k], g, a.scale2, masked, first, p[k].low, p[k].high, 8.0f, sees);
        }
        read(4 * C, x[0]);
        __builtin_amdgcn_sched_barrier(0);
        u32x4 pf[NQ][2];
#pragma unroll
        for (int k = 0; k < NQ; ++k) page_weights<D, DT>(s[k], r[k], pf[k], a.scale2);
#pragma unroll
        for (int f = 0; f < D / 8; f += 4) {
          if (f + 4 < D / 8) read(4 * C + f + 4, x[(f / 4 + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int k = 0; k < NQ; ++k)
              r[k].o[(f + b) >> 1] = KvType<DT>::mfma(x[(f / 4) & 1][b], pf[k][b & 1], r[k].o[(f + b) >> 1]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      page = pn;
      c = cn;
      if (pn >= 0) {
        job.store(frag + (cur ^ 1) * (FRAGS * 64), wave, lane, u.kv - cn * KV_PAGE);
        pn = next_page(cn);
        if (pn >= 0) job.load(heads + pn * page_bytes, wave, lane);
      }
      lds_barrier();
      cur ^= 1;
    }

    const bool whole = n == u.pages;
    const int64_t slot = 2 * (int64_t)wg + (at != share.begin);
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      const float l = row_sum(r[k].l);
      const int in_tile = wave * (NQ * 16) + k * 16 + (lane & 15);
      if (whole) {
        if (in_tile < rows) {
          const float inv = l == 0.0f ? 0.0f : 1.0f / l;
          uint16_t *to = a.out + p[k].t * a.out_token + p[k].hq * a.out_head + g * 4;
#pragma unroll
          for (int ct = 0; ct < D / 16; ++ct) {
            u32x2 x;
            x[0] = KvType<DT>::pack(r[k].o[ct][0] * inv, r[k].o[ct][1] * inv);
            x[1] = KvType<DT>::pack(r[k].o[ct][2] * inv, r[k].o[ct][3] * inv);
            *reinterpret_cast<u32x2 *>(to + ct * 16) = x;
          }
          if (a.lse && g == 0) a.lse[p[k].t * (a.kv_heads * a.group) + p[k].hq] = lse_of(r[k].m, l);
        }
      } else {
        float *to = a.part_o + (slot * TR + in_tile) * D + g * 4;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) *reinterpret_cast<f32x4 *>(to + ct * 16) = r[k].o[ct];
        if (g == 0) {
          a.part_ml[(slot * TR + in_tile) * 2] = r[k].m;
          a.part_ml[(slot * TR + in_tile) * 2 + 1] = l;
        }
      }
    }
    const int next = at + (a.whole ? 1 : n);
    if (tid == 0 && !a.whole && next == share.end) leave_border(a, share, u, wg, at, rows);
    at = next;
  }
  clear_rest<D, THREADS>(a, wg, gridDim.x, tid);
}

// The share that leaves the i-th unit across its border, -1: there are fewer; by the workgroup's 256 threads.
__device__ inline int border_at(const KvAttnArgs &a, int shares, int i, int tid) {
  __shared__ int sums[4], found;
  const int lane = tid & 63, wave = tid >> 6, per = (shares + 255) / 256, first = tid * per, end = min(first + per, shares);
  if (tid == 0) found = -1;
  int own = 0;
#pragma unroll 4
  for (int j = first; j < end; ++j) own += a.borders[(int64_t)j * BORDER_INTS] != 0;
  int x = lanes_up_to(own);
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; ++w) x += sums[w];
  if (i >= x - own && i < x) {
    int left = i - (x - own);
    for (int j = first; j < end; ++j)
      if (a.borders[(int64_t)j * BORDER_INTS] != 0 && left-- == 0) found = j;
  }
  __syncthreads();
  return uniform(found);
}

// Units that several workgroups share.  Workgroup (w, y) adds up the parts of one row (ONE) or some of the unit that goes across
// the border behind share w and began in it; with `shares`, of the w-th such unit of that many shares.  D / 4 lanes have a part (ONE)
// or a row each: decode has one tile of few rows and up to all shares in a unit (520 001 tokens, 64 shares a unit: 40 us with a
// thread a row and 8 channels, now 5), chunks have many rows of few parts (a workgroup a row there: 29 us for 256 shares).
template <int D, int DT, bool ONE>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a, int tile_rows, int shares) {
  constexpr int LANES = D / 4, SETS = 256 / LANES;  // 96 channels: 24 lanes, 10 sets, 16 threads idle
  __shared__ float red_m[4];
  __shared__ f32x4 red_o[ONE ? SETS : 1][LANES];
  __shared__ float red_l[SETS];
  const int tid = threadIdx.x, set = tid / LANES, lane = tid % LANES;
  const int row = ONE ? blockIdx.y : blockIdx.y * SETS + set;
  int border = blockIdx.x;
  if constexpr (ONE) {
    if (shares > 0) border = border_at(a, shares, border, tid);
    if (border < 0) return;
  }
  const int32_t *b = a.borders + (int64_t)border * BORDER_INTS;
  const int n = b[0], late = b[1], t0 = b[2], tile = b[3], head = b[4], rows = b[5];
  if (n == 0 || (ONE ? row : (int)blockIdx.y * SETS) >= rows) return;
  // a workgroup's first unit is in its slot 0
  auto slot = [&](int k) { return 2 * ((int64_t)border + k) + (k == 0 && late); };
  float m = -__builtin_inff(), l = 0.0f;
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (ONE) {
    for (int k = tid; k < n; k += 256) m = fmaxf(m, a.part_ml[(slot(k) * tile_rows + row) * 2]);
    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((tid & 63) == 0) red_m[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
  } else {
    if (set >= SETS || row >= rows) return;
#pragma unroll 4
    for (int k = 0; k < n; ++k) m = fmaxf(m, a.part_ml[(slot(k) * tile_rows + row) * 2]);
  }
  const float base = m == -__builtin_inff() ? 0.0f : m;
  if (set < SETS) {
#pragma unroll 4
    for (int k = ONE ? set : 0; k < n; k += ONE ? SETS : 1) {
      const int64_t at = slot(k) * tile_rows + row;
      const float f = __builtin_amdgcn_exp2f(a.part_ml[at * 2] - base);
      l += f * a.part_ml[at * 2 + 1];
      x += f * *reinterpret_cast<const f32x4 *>(a.part_o + at * D + lane * 4);
    }
  }
  if constexpr (ONE) {
    if (set < SETS) {
      red_o[set][lane] = x;
      if (lane == 0) red_l[set] = l;
    }
    __syncthreads();
    if (set > 0) return;
#pragma unroll
    for (int p = 1; p < SETS; ++p) {
      x += red_o[p][lane];
      l += red_l[p];
    }
  }
  const int i = tile * tile_rows + row;
  const int64_t t = t0 + i / a.group;
  const int hq = head * a.group + i % a.group;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  u32x2 r;
  r[0] = KvType<DT>::pack(x[0] * inv, x[1] * inv);
  r[1] = KvType<DT>::pack(x[2] * inv, x[3] * inv);
  *reinterpret_cast<u32x2 *>(a.out + t * a.out_token + hq * a.out_head + lane * 4) = r;
  if (a.lse && lane == 0) a.lse[t * (a.kv_heads * a.group) + hq] = lse_of(m, l);
}

// How a call is cut: rows of a tile, workgroups, whole units or shares, and the workspace.
struct Shape {
  int tile_rows, n_wg;
  bool whole;
  size_t prefix, borders, ml, o;  // bytes
};

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

Shape shape_of(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_new, int window, int n_select,
               int64_t width) {
  Shape s;
  const int64_t rows = (int64_t)(max_new < tokens ? max_new : tokens) * group;  // of a request and head, at most
  int64_t most = n_select > 0 ? n_select : width;  // pages of a unit
  if (n_select == 0 && window > 0) {
    const int64_t seen = ((int64_t)window + (max_new < tokens ? max_new : tokens)) / KV_PAGE + 2;
    if (seen < most) most = seen;
  }
  // 16 rows a tile up to 64 rows of a request and head (16 requests of 8001 tokens, 64 rows: 91 us, in a tile of the
  // chunks' kernel 95; 64 rows of one of 32 000: 35 and 51; 128 rows go either way: 168 and 108, 49 and 56).  Both are
  // three to five times what reading the pages once takes (28 and 7 us): a page is unpacked for every tile.
  const bool few = n_select > 0 || rows <= 64;
  // Whole units where they are short: 32 requests of 1900 tokens 19 us, in shares and joined 24, 4 requests 15 and 13, one of
  // 334 7.7 and 11; up to twice as long where there are enough of them: 32 requests of 3900 30 us and 36, 4 requests 24 and 16.  Just beyond,
  // requests of one length still gain (32 of 5000: 34 and 39, 64 of 8000: 103 and 107) or not (16 of 5000: 32 and 28); shares
  // have them, as ragged ones leave whole units waiting for the longest.
  const bool narrow = most <= WHOLE_PAGES || (few && most <= 2 * WHOLE_PAGES && tokens * kv_heads >= 128);
  // Chunks: tiles of 256 rows where they fill the CUs (a page is unpacked by twice the wavefronts: 2048 tokens,
  // 32 heads, behind 8190: 331 us, 128 rows 379; 4 x 700 behind 2000: 162 and 172), of 128 otherwise, and of 64 where units
  // are short, so that shares cannot fill the chip instead (1700 tokens, 16 heads of their own keys, a window of 1000:
  // 38 us, 128 rows 44; 3 x 300, 8 heads: 32 and 44; 4 x 200, 8 heads of two, no window: 23 and 30; 2 x 400, 8 heads of four,
  // a window of 1500: 47 and 48).  256 channels have no registers for more than 16 rows a wavefront.
  const int64_t all = tokens * group * kv_heads;
  s.tile_rows = few ? 16 : D == 256 ? 128 : all >= 256 * 256 ? 256 : narrow && all < 512 * 128 ? 64 : 128;
  const int64_t units = n_select > 0 ? tokens * kv_heads * ((group + 15) / 16)
                                     : (tokens * group / s.tile_rows + requests) * kv_heads;
  // whole units where they are short, or (chunks) where there are many; shares otherwise: as many workgroups as the
  // chip holds at a time, four pages each at least
  const int fill = s.tile_rows == 16 ? 512 : s.tile_rows == 128 && D < 256 ? 512 : 256;
  const bool units_fit = narrow || (s.tile_rows > 16 && units >= 1024);
  // (and where their pages cannot be counted in 31 bits, whatever max_new promises)
  const int64_t surely = n_select > 0 ? n_select : window > 0 ? (window + tokens) / KV_PAGE + 2 : width;
  s.whole = units_fit || units * (n_select > 0 || surely < width ? surely : width) > 0x7fffffff;
  const int shares = units * most / 4 >= fill ? fill : (int)(units * most / 4 + 1);
  s.n_wg = s.whole ? (int)units : shares;
  if (s.n_wg < 1) s.n_wg = 1;
  // Room for shares also where only the 31 bits forbid them: a window may lift that, and what is asked for without one has
  // to be enough.
  s.prefix = up256((size_t)(requests + 1) * 4);
  s.borders = units_fit ? 0 : up256((size_t)shares * BORDER_INTS * 4);
  s.ml = units_fit ? 0 : up256((size_t)shares * 2 * s.tile_rows * 2 * 4);
  s.o = units_fit ? 0 : up256((size_t)shares * 2 * s.tile_rows * D * 4);
  return s;
}

template <typename K>
int allow_lds(K kernel, size_t lds) {
  if (lds > 65536)
    KV_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  return IVFPQ_OK;
}

template <int D, int DT, bool TREE>
int attention_of(KvAttnArgs a, const Shape &sh, hipStream_t s) {
  const bool sel = a.selected != nullptr;
  a.scanned = !sel && a.requests > SCAN_REQUESTS;
  if (a.scanned) {
    hipLaunchKernelGGL(kv_scan_kernel, dim3(1), dim3(1024), 0, s, a, sh.tile_rows, 0);
    KV_HIP_TRY(hipGetLastError());
  }
  const size_t lists = sel || a.scanned ? 0 : ((size_t)a.requests + 3 * (size_t)(a.requests + 1)) * 4;
  int rc;
  if (sh.tile_rows == 16) {
    const size_t lds = (size_t)(4 * 16 * (D + 4) + 4 * 16 * 2) * 4 + 4 * 4 + lists;
    auto rows16 = [&](auto SEL) -> int {
      constexpr bool select = decltype(SEL)::value;
      if ((rc = allow_lds(&kv_rows16_kernel<D, DT, select, TREE>, lds))) return rc;
      hipLaunchKernelGGL((kv_rows16_kernel<D, DT, select, TREE>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
      return IVFPQ_OK;
    };
    if constexpr (TREE) rc = rows16(std::false_type());  // (a tree's tokens have no selected pages)
    else rc = sel ? rows16(std::true_type()) : rows16(std::false_type());
    if (rc) return rc;
  } else {
    const size_t lds = (size_t)2 * page_fragments<D>() * 1024 + 8 * 4 + lists;
    if constexpr (D == 256) {
      if ((rc = allow_lds(&kv_rows_kernel<D, DT, 8, 1, TREE>, lds))) return rc;
      hipLaunchKernelGGL((kv_rows_kernel<D, DT, 8, 1, TREE>), dim3((unsigned)a.n_wg), dim3(512), lds, s, a);
    } else if (sh.tile_rows == 256) {
      if ((rc = allow_lds(&kv_rows_kernel<D, DT, 8, 2, TREE>, lds))) return rc;
      hipLaunchKernelGGL((kv_rows_kernel<D, DT, 8, 2, TREE>), dim3((unsigned)a.n_wg), dim3(512), lds, s, a);
    } else if (sh.tile_rows == 64) {
      if ((rc = allow_lds(&kv_rows_kernel<D, DT, 4, 1, TREE>, lds))) return rc;
      hipLaunchKernelGGL((kv_rows_kernel<D, DT, 4, 1, TREE>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
    } else {
      if ((rc = allow_lds(&kv_rows_kernel<D, DT, 4, 2, TREE>, lds))) return rc;
      hipLaunchKernelGGL((kv_rows_kernel<D, DT, 4, 2, TREE>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
    }
  }
  KV_HIP_TRY(hipGetLastError());
  if (a.whole || a.n_wg == 1) return IVFPQ_OK;
  const int64_t most = a.tokens * (int64_t)a.group;
  if (sh.tile_rows == 16) {
    const int rows = (int)(sel && a.group < 16 ? a.group : most < 16 ? most : 16);
    hipLaunchKernelGGL((kv_join_kernel<D, DT, true>), dim3((unsigned)(a.n_wg - 1), (unsigned)rows), dim3(256), 0, s, a, 16, 0);
  } else {
    constexpr int SETS = 256 / (D / 4);
    hipLaunchKernelGGL((kv_join_kernel<D, DT, false>), dim3((unsigned)(a.n_wg - 1), (unsigned)((sh.tile_rows + SETS - 1) / SETS)),
                       dim3(256), 0, s, a, sh.tile_rows, 0);
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

void place_workspace(KvAttnArgs &a, const Shape &sh, char *workspace) {
  a.n_wg = sh.n_wg;
  a.whole = sh.whole;
  a.prefix = reinterpret_cast<int32_t *>(workspace);
  a.borders = reinterpret_cast<int32_t *>(workspace + sh.prefix);
  a.part_ml = reinterpret_cast<float *>(workspace + sh.prefix + sh.borders);
  a.part_o = reinterpret_cast<float *>(workspace + sh.prefix + sh.borders + sh.ml);
}

}  // namespace

}  // namespace ivfpq

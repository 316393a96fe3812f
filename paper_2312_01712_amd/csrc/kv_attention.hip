// Attention of a step's new tokens over the paged 4-bit cache, all pages or selected ones.
//
// The running form of the softmax: with s_j = scale log2(e) q . k_j, a row keeps m = max s_j,
// l = sum 2^(s_j - m) and o = sum 2^(s_j - m) v_j and multiplies l and o by 2^(m_old - m_new) when m
// grows; parts of the keys joined the same way.  Sums and statistics are in 32 bits, weights are
// rounded to the cache's type for the second product (as the values are: both factors exact or
// within half a unit of the result's type).
//
// Layout.  A wavefront has 16 rows (query heads of one kv head, tokens above them) and works on
// S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's statistics and the exponentials
// of the first product are, in place, the second operand of the second: lane (g, row) has keys
// 16 tt + 4 g + i, and the page stores the values in this order of tokens.

#include <type_traits>

#include "kv_internal.h"

namespace ivfpq {

namespace {

constexpr int SCAN_REQUESTS = 2048;  // more than these: their units are scanned by a launch of its own

__device__ inline float xor16_max(float x) { return fmaxf(x, __shfl_xor(x, 16)); }
__device__ inline float xor32_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }

// values that are the same in all lanes, in scalar registers
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// pages [lo, lo + n) that any new token of a request sees; n >= 1
struct Range {
  int lo, n;
};

// What a workgroup leaves about the unit that goes across the border behind its share, if it began in it:
// shares that have some of it (0: there is none), whether it is not the first unit in its first
// share, first token, tile, kv head, rows.
constexpr int BORDER_INTS = 8;

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

template <int D, int DT>
__device__ inline void page_values(const Page<D> &pg, const u32x4 *pf, f32x4 *o) {
#pragma unroll
  for (int p = 0; p < D / 32; ++p)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 lo, hi;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t w = pg.v[p][u * 2 + half], sc = pg.vs[p][u * 2 + half];
        const uint32_t a = unpack_v<DT, 0>(w, sc), b = unpack_v<DT, 1>(w, sc), c = unpack_v<DT, 2>(w, sc),
                       d = unpack_v<DT, 3>(w, sc);
        lo[half * 2] = __builtin_amdgcn_perm(b, a, 0x05040100);
        hi[half * 2] = __builtin_amdgcn_perm(b, a, 0x07060302);
        lo[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x05040100);
        hi[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x07060302);
      }
      o[2 * p] = KvType<DT>::mfma(lo, pf[u], o[2 * p]);
      o[2 * p + 1] = KvType<DT>::mfma(hi, pf[u], o[2 * p + 1]);
    }
}

// One page into the rows.  first: position of the page's first key; the row sees (low, high].
template <int D, int DT>
__device__ inline void page_step(const Page<D> &pg, const u32x4 *qf, Row<D> &r, int lane, float scale2, bool masked,
                                 int first, int low, int high) {
  f32x4 s[4];
  page_scores<D, DT>(pg, qf, lane, s);
  float top = -__builtin_inff();
#pragma unroll
  for (int tt = 0; tt < 4; ++tt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[tt][i] *= scale2;
      if (masked) {
        const int j = first + tt * 16 + (lane >> 4) * 4 + i;
        s[tt][i] = j > low && j <= high ? s[tt][i] : -__builtin_inff();
      }
      top = fmaxf(top, s[tt][i]);
    }
  top = xor32_max(xor16_max(top));
  const float m = fmaxf(r.m, top);
  if (__any(m > r.m)) {
    const float f = m > r.m ? __builtin_amdgcn_exp2f(r.m - m) : 1.0f;
    r.l *= f;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) r.o[ct][i] *= f;
    r.m = m;
  }
  const float base = m == -__builtin_inff() ? 0.0f : m;  // a row that saw nothing so far: every weight is 0
  u32x4 pf[2];
#pragma unroll
  for (int tt = 0; tt < 4; ++tt) {
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e[i] = __builtin_amdgcn_exp2f(s[tt][i] - base);
      r.l += e[i];
    }
    pf[tt >> 1][(tt & 1) * 2] = KvType<DT>::pack(e[0], e[1]);
    pf[tt >> 1][(tt & 1) * 2 + 1] = KvType<DT>::pack(e[2], e[3]);
  }
  page_values<D, DT>(pg, pf, r.o);
}

template <int DT>
__device__ inline void store_row(uint16_t *to, const float *x, int n) {
  for (int c = 0; c < n; c += 2) *reinterpret_cast<uint32_t *>(to + c) = KvType<DT>::pack(x[c], x[c + 1]);
}

// Rows of a unit: row i of tile `tile` of a group is token i / G, head i % G (of the kv head); with
// selected pages a group is one token.
struct Unit {
  int g, head, tile, lo, pages;  // group, kv head, tile of 16 rows, first page (or list entry), pages
  int t0, fresh, kv, req;        // first token, tokens, held, request
  int64_t first;                 // index of its first page among all units' pages
};

template <int D, int DT, bool SEL>
__device__ inline void join_waves(const KvAttnArgs &a, const Unit &u, int rows, bool whole, int64_t slot, float (*ml)[16][2],
                                  float *buf, int tid) {
  // buf [4][16][D + 4], ml [4]
  const int row = tid >> 4, part = tid & 15;
  float m = -__builtin_inff(), l = 0.0f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w][row][0]);
  const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(ml[w][row][0] - base);
    l += f[w] * ml[w][row][1];
  }
  float x[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    x[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) x[c] += f[w] * buf[(w * 16 + row) * (D + 4) + part * (D / 16) + c];
  }
  if (whole) {
    if (row < rows) {
      const int i = u.tile * 16 + row;
      const int64_t t = u.t0 + i / a.group;
      const int hq = u.head * a.group + i % a.group;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) x[c] *= inv;
      store_row<DT>(a.out + t * a.out_token + hq * a.out_head + part * (D / 16), x, D / 16);
      if (a.lse && part == 0)
        a.lse[t * (a.kv_heads * a.group) + hq] =
            l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
    }
  } else {
    float *to = a.part_o + (slot * 16 + row) * D + part * (D / 16);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) to[c] = x[c];
    if (part == 0) {
      a.part_ml[(slot * 16 + row) * 2] = m;
      a.part_ml[(slot * 16 + row) * 2 + 1] = l;
    }
  }
}

// rows that stand for no token: behind the last request's tokens
template <int D>
__device__ inline void clear_rest(const KvAttnArgs &a, int64_t wg, int64_t n_wg, int tid) {
  const int heads = a.kv_heads * a.group;
  int64_t t = a.requests > 0 ? a.q_start[a.requests] : 0;
  if (t < 0) t = 0;
  const int64_t n = (a.tokens - t) * heads;
  for (int64_t i = wg * 256 + tid; i < n * (D / 8); i += n_wg * 256) {
    const int64_t row = i / (D / 8);
    *reinterpret_cast<u32x4 *>(a.out + (t + row / heads) * a.out_token + (row % heads) * a.out_head + (i % (D / 8)) * 8) =
        u32x4{0, 0, 0, 0};
    if (a.lse && i % (D / 8) == 0) a.lse[t * heads + row] = -__builtin_inff();
  }
}

// Which group a unit of pages belongs to.  Dense: groups are requests and `prefix` holds the units
// before each; selected: every token has the same number.
template <bool SEL>
__device__ inline Unit unit_at(const KvAttnArgs &a, const int64_t *prefix, int64_t at, int64_t &offset) {
  Unit u;
  if constexpr (SEL) {
    const int tiles = (a.group + 15) / 16;
    const int64_t per = (int64_t)a.kv_heads * tiles * a.n_select;
    u.g = (int)(at / per);
    const int64_t rest = at % per, k = rest / a.n_select;
    u.head = (int)(k / tiles), u.tile = (int)(k % tiles);
    u.lo = 0, u.pages = a.n_select;
    offset = rest % a.n_select;
    u.t0 = u.g, u.fresh = 1;
    const int r = uniform(a.token_req[u.g]);
    u.req = (uint32_t)r < (uint32_t)a.requests ? r : -1;
    u.kv = u.req >= 0 ? uniform(a.kv_lens[u.req]) : 0;
  } else {
    int lo = 0, hi = a.requests;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (uniform(prefix[mid]) <= at) lo = mid;
      else hi = mid;
    }
    u.g = u.req = lo;
    u.t0 = uniform(a.q_start[lo]);
    u.fresh = min(uniform(a.q_start[lo + 1]), a.tokens) - u.t0;
    u.kv = uniform(a.kv_lens[lo]);
    const Range pr = request_pages(u.kv, u.fresh, a.window, a.width);
    const int tiles = (int)(((int64_t)u.fresh * a.group + 15) / 16);
    const int64_t rest = at - uniform(prefix[lo]), k = rest / pr.n;
    u.head = (int)(k / tiles), u.tile = (int)(k % tiles);
    u.lo = pr.lo, u.pages = pr.n;
    offset = rest % pr.n;
  }
  u.first = at - offset;
  return u;
}

__device__ inline int64_t units_of(const KvAttnArgs &a, int g) {
  const int fresh = min(a.q_start[g + 1], a.tokens) - a.q_start[g];
  if (fresh <= 0) return 0;
  return (((int64_t)fresh * a.group + 15) / 16) * a.kv_heads * request_pages(a.kv_lens[g], fresh, a.window, a.width).n;
}

// Units before every group, by the whole workgroup; returns their sum.
__device__ inline int64_t scan_units(const KvAttnArgs &a, int64_t *prefix, int64_t *sums, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  int64_t carry = 0;
  for (int b = 0; b < a.requests; b += 256) {
    const int64_t n = b + tid < a.requests ? units_of(a, b + tid) : 0;
    int64_t x = n;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += sums[w];
    if (b + tid < a.requests) prefix[b + tid] = carry + x - n;
    carry += sums[0] + sums[1] + sums[2] + sums[3];
  }
  __syncthreads();
  return carry;
}

__global__ __launch_bounds__(256) void kv_scan_kernel(KvAttnArgs a) {
  __shared__ int64_t sums[4];
  const int64_t total = scan_units(a, a.prefix, sums, threadIdx.x);
  if (threadIdx.x == 0) a.prefix[a.requests] = total;
}

// A workgroup has an equal share of all (group, head, tile, page) units, in this order: ragged
// requests cost no balance.  Its four wavefronts take the share's pages in turn, each with its own
// softmax state; what a workgroup has of a unit whose pages it does not have all goes to the
// workspace, and kv_join_kernel adds up.
// Bound by reading the pages (decode: 16 rows or fewer share a page).
template <int D, int DT, bool SEL>
__global__ __launch_bounds__(256, 2) void kv_rows16_kernel(KvAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float *buf = reinterpret_cast<float *>(lds);                                     // [4][16][D + 4]
  float(*ml)[16][2] = reinterpret_cast<float(*)[16][2]>(buf + 4 * 16 * (D + 4));  // [4]
  int64_t *sums = reinterpret_cast<int64_t *>(ml + 4);                            // [4]
  int64_t *own_prefix = sums + 4;                                                 // [requests], dense
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4;
  const int64_t wg = blockIdx.x;

  clear_rest<D>(a, wg, gridDim.x, tid);
  int64_t total;
  if constexpr (SEL) total = (int64_t)(a.requests > 0 ? min(a.q_start[a.requests], a.tokens) : 0) * a.kv_heads * ((a.group + 15) / 16) * a.n_select;
  else total = a.scanned ? a.prefix[a.requests] : scan_units(a, own_prefix, sums, tid);
  const int64_t *prefix = !SEL && a.scanned ? a.prefix : own_prefix;
  total = uniform(total);
  int64_t span = (total + a.n_wg - 1) / a.n_wg;
  if (span < 4) span = 4;
  const int64_t begin = wg * span, end = min(begin + span, total);
  if (tid == 0 && begin >= end) a.borders[wg * BORDER_INTS] = 0;
  for (int64_t at = begin; at < end;) {
    int64_t offset;
    const Unit u = unit_at<SEL>(a, prefix, at, offset);
    const int n = (int)min((int64_t)u.pages - offset, end - at);
    const int rows = min(16, u.fresh * a.group - u.tile * 16);
    // the lane's row
    const int i = u.tile * 16 + min(lane & 15, rows - 1);
    const int64_t t = u.t0 + i / a.group;
    const int hq = u.head * a.group + i % a.group;
    const int pos = a.positions[t];
    const int high = min(pos, u.kv - 1), low = a.window > 0 ? pos - a.window : -1;
    // over the wavefront: keys below `clear_high` and above `clear_low` are seen by every row
    int clear_high = high, clear_low = low, any_high = high, any_low = low;
    for (int d = 1; d < 16; d <<= 1) {
      clear_high = min(clear_high, __shfl_xor(clear_high, d));
      any_high = max(any_high, __shfl_xor(any_high, d));
      clear_low = max(clear_low, __shfl_xor(clear_low, d));
      any_low = min(any_low, __shfl_xor(any_low, d));
    }
    clear_high = uniform(clear_high);
    clear_low = uniform(clear_low);
    any_high = uniform(any_high);
    any_low = uniform(any_low);
    u32x4 qf[D / 32];
    {
      const uint16_t *qp = a.q + t * a.q_token + hq * a.q_head + g * (D / 4);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[c] = *reinterpret_cast<const u32x4 *>(qp + c * 8);
    }
    Row<D> r;
    r.m = -__builtin_inff();
    r.l = 0.0f;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) r.o[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int32_t *table = a.table + (int64_t)max(u.req, 0) * a.width;
    const int32_t *list = SEL ? a.selected + ((int64_t)u.t0 * a.kv_heads + u.head) * a.n_select : nullptr;
    const char *heads = a.pages + u.head * (int64_t)kv_head_bytes(D);
    const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
    const int k1 = (int)offset + n;
    // the wavefront's entries offset + wave, + 4, ...: a lane looks 64 of them up at a time
    for (int k0 = (int)offset + wave; k0 < k1; k0 += 4 * 64) {
      const int k = k0 + 4 * lane;
      int c = -1, page = -1;
      if (k < k1 && u.req >= 0) {
        c = u.lo + k;
        if constexpr (SEL) c = list[k];
        // a column that no row sees anything of, or without a page in the cache
        if ((uint32_t)c < (uint32_t)a.width && c * KV_PAGE <= any_high && c * KV_PAGE + KV_PAGE - 1 > any_low) page = table[c];
      }
      uint64_t todo = __ballot((uint32_t)page < (uint64_t)a.n_pages);
      auto fetch = [&](Page<D> &pg, uint64_t left) {
        pg.load(heads + __builtin_amdgcn_readlane(page, __builtin_ctzll(left)) * page_bytes, lane);
      };
      auto step = [&](Page<D> &pg, uint64_t left) {
        const int first = __builtin_amdgcn_readlane(c, __builtin_ctzll(left)) * KV_PAGE;
        if (first + KV_PAGE > u.kv) pg.cut(u.kv - first, lane);
        const bool masked = first + KV_PAGE - 1 > clear_high || first <= clear_low;
        page_step<D, DT>(pg, qf, r, lane, a.scale2, masked, first, low, high);
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
    // l of the whole row
    r.l += __shfl_xor(r.l, 16);
    r.l += __shfl_xor(r.l, 32);
    __syncthreads();  // the buffer is free again
    if (g == 0) ml[wave][lane & 15][0] = r.m, ml[wave][lane & 15][1] = r.l;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
      *reinterpret_cast<f32x4 *>(buf + (wave * 16 + (lane & 15)) * (D + 4) + ct * 16 + g * 4) = r.o[ct];
    __syncthreads();
    join_waves<D, DT, SEL>(a, u, rows, n == u.pages, 2 * wg + (at != begin), ml, buf, tid);
    if (tid == 0 && at + n == end) {
      const bool across = u.first + u.pages > end && u.first >= begin;
      int32_t *b = a.borders + wg * BORDER_INTS;
      b[0] = across ? (int32_t)((u.first + u.pages - 1) / span - wg) + 1 : 0;
      b[1] = at != begin;
      b[2] = u.t0;
      b[3] = u.tile;
      b[4] = u.head;
      b[5] = rows;
    }
    at += n;
  }
}

// Units that several workgroups share.  Workgroup (w, row) adds up one row's parts of the unit that goes across
// the border behind share w and began in it.  D / 4 lanes have a part each, so that a context that the whole chip shares is joined in
// a few trips to memory (520 001 tokens, 64 shares a unit: 40 us with a thread a row and 8 channels, now 4).
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a) {
  constexpr int LANES = D / 4, PARTS = 256 / LANES;  // 96 channels: 24 lanes, 10 parts, 16 threads idle
  __shared__ float red_m[4];
  __shared__ f32x4 red_o[PARTS][LANES];
  __shared__ float red_l[PARTS];
  const int tid = threadIdx.x, row = blockIdx.y;
  const int32_t *b = a.borders + (int64_t)blockIdx.x * BORDER_INTS;
  const int n = b[0], late = b[1], t0 = b[2], tile = b[3], head = b[4], rows = b[5];
  if (n == 0 || row >= rows) return;
  // a workgroup's first unit is in its slot 0
  auto slot = [&](int k) { return 2 * ((int64_t)blockIdx.x + k) + (k == 0 && late); };
  float m = -__builtin_inff();
  for (int k = tid; k < n; k += 256) m = fmaxf(m, a.part_ml[(slot(k) * 16 + row) * 2]);
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((tid & 63) == 0) red_m[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
  const float base = m == -__builtin_inff() ? 0.0f : m;
  const int part = tid / LANES, lane = tid % LANES;
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  float l = 0.0f;
  if (part < PARTS) {
#pragma unroll 4
    for (int k = part; k < n; k += PARTS) {
      const int64_t at = slot(k) * 16 + row;
      const float f = __builtin_amdgcn_exp2f(a.part_ml[at * 2] - base);
      l += f * a.part_ml[at * 2 + 1];
      x += f * *reinterpret_cast<const f32x4 *>(a.part_o + at * D + lane * 4);
    }
    red_o[part][lane] = x;
    if (lane == 0) red_l[part] = l;
  }
  __syncthreads();
  if (part > 0) return;
#pragma unroll
  for (int p = 1; p < PARTS; ++p) {
    x += red_o[p][lane];
    l += red_l[p];
  }
  const int i = tile * 16 + row;
  const int64_t t = t0 + i / a.group;
  const int hq = head * a.group + i % a.group;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  u32x2 r;
  r[0] = KvType<DT>::pack(x[0] * inv, x[1] * inv);
  r[1] = KvType<DT>::pack(x[2] * inv, x[3] * inv);
  *reinterpret_cast<u32x2 *>(a.out + t * a.out_token + hq * a.out_head + lane * 4) = r;
  if (a.lse && lane == 0)
    a.lse[t * (a.kv_heads * a.group) + hq] = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

template <int D, int DT, bool SEL>
int attention_of(KvAttnArgs a, hipStream_t s) {
  a.scanned = !SEL && a.requests > SCAN_REQUESTS;
  if (a.scanned) {
    hipLaunchKernelGGL(kv_scan_kernel, dim3(1), dim3(256), 0, s, a);
    KV_HIP_TRY(hipGetLastError());
  }
  const size_t lds = (size_t)(4 * 16 * (D + 4) + 4 * 16 * 2) * 4 + 4 * 8 + (SEL || a.scanned ? 0 : (size_t)a.requests * 8);
  if (lds > 65536) KV_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_rows16_kernel<D, DT, SEL>),
                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  hipLaunchKernelGGL((kv_rows16_kernel<D, DT, SEL>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
  KV_HIP_TRY(hipGetLastError());
  if (a.n_wg == 1) return IVFPQ_OK;
  const int rows = (int)(a.tokens * (int64_t)a.group < 16 ? a.tokens * (int64_t)a.group : !SEL || a.group > 16 ? 16 : a.group);
  hipLaunchKernelGGL((kv_join_kernel<D, DT>), dim3((unsigned)(a.n_wg - 1), (unsigned)rows), dim3(256), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

template <int D>
int attention_typed(const KvAttnArgs &a, int dtype, hipStream_t s) {
  if (dtype == IVFPQ_KV_BF16)
    return a.selected ? attention_of<D, IVFPQ_KV_BF16, true>(a, s) : attention_of<D, IVFPQ_KV_BF16, false>(a, s);
  return a.selected ? attention_of<D, IVFPQ_KV_FP16, true>(a, s) : attention_of<D, IVFPQ_KV_FP16, false>(a, s);
}

struct Shape {
  int64_t units;   // (group, head, tile), at most
  int n_wg;
  size_t prefix, borders, ml, o;  // bytes
};

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

Shape shape_of(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int n_select, int64_t width) {
  Shape s;
  s.units = n_select > 0 ? tokens * kv_heads * ((group + 15) / 16) : (tokens * group / 16 + requests) * kv_heads;
  const int64_t pages = s.units * (n_select > 0 ? n_select : width);
  // two workgroups on every CU, four pages each at least
  s.n_wg = pages / 4 >= 512 ? 512 : (int)(pages / 4 + 1);
  s.prefix = up256((size_t)(requests + 1) * 8);
  s.borders = up256((size_t)s.n_wg * BORDER_INTS * 4);
  s.ml = up256((size_t)s.n_wg * 2 * 16 * 2 * 4);
  s.o = up256((size_t)s.n_wg * 2 * 16 * D * 4);
  return s;
}

}  // namespace

size_t kv_attention_workspace(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_new, int n_select,
                              int64_t width) {
  (void)max_new;
  const Shape s = shape_of(tokens, requests, kv_heads, group, D, n_select, width);
  return s.prefix + s.borders + s.ml + s.o;
}

int launch_kv_attention(KvAttnArgs a, int D, int dtype, int max_new, char *workspace, hipStream_t s) {
  (void)max_new;
  const Shape sh = shape_of(a.tokens, a.requests, a.kv_heads, a.group, D, a.selected ? a.n_select : 0, a.width);
  a.n_wg = sh.n_wg;
  a.prefix = reinterpret_cast<int64_t *>(workspace);
  a.borders = reinterpret_cast<int32_t *>(workspace + sh.prefix);
  a.part_ml = reinterpret_cast<float *>(workspace + sh.prefix + sh.borders);
  a.part_o = reinterpret_cast<float *>(workspace + sh.prefix + sh.borders + sh.ml);
  switch (D) {
    case 64: return attention_typed<64>(a, dtype, s);
    case 96: return attention_typed<96>(a, dtype, s);
    case 128: return attention_typed<128>(a, dtype, s);
    default: return attention_typed<256>(a, dtype, s);
  }
}

}  // namespace ivfpq

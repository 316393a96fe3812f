// Attention of drafted tokens over the paged 4-bit cache: what is held before them, and of themselves what their masks say.
//
// The kernels of kv_attention_kernels.h with masks, and one of its own for trees of some tokens: two to four tiles of 16 rows for a kv
// head are too many for the kernel of decoding, which unpacks a page for every tile, and too few for that of chunks, which unpacks
// pages into LDS for many.  Here a wavefront has pages of its own, as in decoding, but every fragment that it unpacks feeds the
// products of two tiles.  Pages come into LDS without passing registers, so that three wavefronts fit a SIMD.

#include "kv_attention_kernels.h"

namespace ivfpq {

namespace {

constexpr int NT = 2;  // tiles of 16 rows of a unit

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

// All N tiles' rows, those behind the unit's last as that one: what is done with them is not kept, but their masks are looked at.
template <int D, int N>
__device__ inline void place_rows(const KvAttnArgs &a, const Unit &u, int rows, RowsInLds<D> &to, int tid) {
  const uint32_t flip = a.negative ? 0x80008000u : 0u;  // a negative scale: of the rows' values
  for (int job = tid; job < N * 16 * (D / 8); job += 256) {
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

// As unpack_tokens.
template <int DT>
__device__ inline void four_tokens(uint32_t w, uint32_t sc, u32x4 &lo, u32x4 &hi, int half) {
  const uint32_t a = KvType<DT>::template unpack<0>(w, scale_byte<0>(sc)), b = KvType<DT>::template unpack<1>(w, scale_byte<1>(sc));
  const uint32_t c = KvType<DT>::template unpack<2>(w, scale_byte<2>(sc)), d = KvType<DT>::template unpack<3>(w, scale_byte<3>(sc));
  lo[half * 2] = __builtin_amdgcn_perm(b, a, 0x05040100);
  hi[half * 2] = __builtin_amdgcn_perm(b, a, 0x07060302);
  lo[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x05040100);
  hi[half * 2 + 1] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

// A unit's rows, N tiles of 16, over the wavefront's part of its pages [offset, offset + n): entries offset + wave, + 4, ...  Keys and
// values of a page have a place each in LDS, of the wavefront alone; the next page's are requested as soon as these are used.
template <int D, int DT, int N>
__device__ inline void tiles_pages(const KvAttnArgs &a, const Unit &u, int rows, int offset, int n, int wave, int lane, int tid,
                                   RowsInLds<D> &in, char *place, Row<D> *r) {
  constexpr int C = D / 32, LOADS = half_loads<D>();
  constexpr float SLACK = 8.0f, LIFT = DT == IVFPQ_KV_FP16 ? 15.0f - SLACK : 0.0f;
  const int row = lane & 15, g = lane >> 4;
  const int32_t *table = a.table + (int64_t)u.req * a.width;
  const char *heads = a.pages + u.head * (int64_t)kv_head_bytes(D);
  const int64_t page_bytes = a.kv_heads * (int64_t)kv_head_bytes(D);
  const int past = min(u.pos0, u.kv);
  // what no row sees less than, and none more (as positions do not follow the order of tokens)
  const int any_low = a.window > 0 ? u.pos0 - a.window : -1, clear_low = a.window > 0 ? u.pos0 + u.fresh - 1 - a.window : -1;

  int k0 = offset + wave, numbers = -1;
  const int k1 = offset + n;
  uint64_t todo = 0;
  auto look = [&]() {  // 64 entries at a time, a lane each
    const int k = k0 + 4 * lane, c = u.lo + k;
    numbers = k < k1 && c < a.width && c * KV_PAGE < u.kv && c * KV_PAGE + KV_PAGE - 1 > any_low ? table[c] : -1;
    todo = __ballot((uint32_t)numbers < (uint64_t)a.n_pages);
  };
  auto next_page = [&](int &first) -> int {
    while (!todo) {
      k0 += 4 * 64;
      if (k0 >= k1) return -1;
      look();
    }
    const int j = __builtin_ctzll(todo);
    todo &= todo - 1;
    first = (u.lo + k0 + 4 * j) * KV_PAGE;
    return __builtin_amdgcn_readlane(numbers, j);
  };
  if (k0 < k1) look();
  int first = 0, page = next_page(first);
  char *keys = place, *values = place + half_bytes<D>();
  if (page >= 0) {
    fetch_half<D>(heads + page * page_bytes, keys, lane);
    fetch_half<D>(heads + page * page_bytes + 34 * D, values, lane);
  }
  place_rows<D, N>(a, u, rows, in, tid);
  __syncthreads();

  while (page >= 0) {
    int first_next = 0;
    const int page_next = next_page(first_next);
    wait_loads<LOADS>();  // the keys are there
    const bool masked = first + KV_PAGE > past || first <= clear_low;
    u32x4 pf[N][2];
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
        for (int k = 0; k < N; ++k) q[k] = *reinterpret_cast<const u32x4 *>(&in.query[k * 16 + row][g * (D / 4) + c * 8]);
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
          const uint64_t sees = tree_sees(a, u, in.token[k * 16 + row], in.low[k * 16 + row], first) >> (4 * g);
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
#pragma unroll
    for (int v = 0; v < C; ++v) {
      const u32x4 w = *reinterpret_cast<const u32x4 *>(values + v * 1024 + lane * 16);
      const u32x4 sc = *reinterpret_cast<const u32x4 *>(values + 32 * D + v * 64 + g * 16);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 lo, hi;
#pragma unroll
        for (int half = 0; half < 2; ++half) four_tokens<DT>(w[h * 2 + half], sc[h * 2 + half], lo, hi, half);
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

// Units of up to NT tiles, shared out among workgroups as in kv_rows16_kernel; a workgroup's four wavefronts take a unit's pages in
// turn and add up through LDS.  Bound by the issue of instructions (vector units 53 % busy, matrix units 23 %, and a product takes the
// issue of seven cycles): a page and two tiles are 420 instructions of the vector units, half of them unpacking, and 64 products.  16
// tokens of 32 heads behind 300 001, 79 GFLOP, 328 MB, 117 us and 10 of joining (16 rows a tile as in decoding: 168 in all); trees
// of up to 32 tokens, 64 heads, behind 24 contexts to 33 000, 117 GFLOP, 190 us (in the kernel of chunks 245).  Three tiles with two
// wavefronts a SIMD took 160 and 282 us, four, which leave a few values to memory in the loop, 169 and 328.  Scaled products of the 4-bit
// codes themselves would save unpacking keys, but sum to 2^-17 of the sizes' sum only, and take no 16-bit queries.
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
    total = scan_units<TR, 256>(a, q, sums, tid);
  }
  const Share share = share_of(a, total, wg);
  if (tid == 0 && !a.whole && share.begin >= share.end) a.borders[(int64_t)wg * BORDER_INTS] = 0;
  for (int at = share.begin; at < share.end;) {
    int offset;
    Unit u = unit_at<TR, false>(a, q, at, offset);
    // entries of the unit: unit_extra, then its pages
    const int extra = a.whole ? 0 : unit_extra<TR>(), entries = u.pages + extra;
    const int taken = a.whole ? entries : min(entries - offset, share.end - at);
    const int first = max(offset - extra, 0), n = max(offset + taken - extra, 0) - first;
    const int rows = min(TR, u.fresh * a.group - u.tile * TR);
    Row<D> r[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      r[k].m = -__builtin_inff();
      r[k].l = 0.0f;
#pragma unroll
      for (int ct = 0; ct < D / 16; ++ct) r[k].o[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int tiles = (rows + 15) / 16;
    char *place = lds + wave * (2 * half_bytes<D>());
    if (tiles == 1) tiles_pages<D, DT, 1>(a, u, rows, first, n, wave, lane, tid, in, place, r);
    else tiles_pages<D, DT, NT>(a, u, rows, first, n, wave, lane, tid, in, place, r);
#pragma unroll
    for (int k = 0; k < NT; ++k)
      if (k < tiles) {
        r[k].l = row_sum(r[k].l);
        __syncthreads();  // the pages are used, or the buffer is free again
        if (g == 0) ml[wave][lane & 15][0] = r[k].m, ml[wave][lane & 15][1] = r[k].l;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct)
          *reinterpret_cast<f32x4 *>(buf + (wave * 16 + (lane & 15)) * (D + 4) + ct * 16 + g * 4) = r[k].o[ct];
        __syncthreads();
        join_waves<D, DT, NT>(a, u, rows, taken == entries, 2 * (int64_t)wg + (at != share.begin), ml, buf, tid, k);
      }
    __syncthreads();
    const int next = at + (a.whole ? 1 : taken);
    u.pages = entries;
    if (tid == 0 && !a.whole && next == share.end) leave_border(a, share, u, wg, at, rows);
    at = next;
  }
  clear_rest<D, 256>(a, wg, gridDim.x, tid);
}

// How a call is cut.  tiles: of 16 rows that a wavefront has, or 0 for the kernels of chunks.
struct TreeShape : Shape {
  int tiles;
  int64_t units;
};

TreeShape tree_shape(int64_t tokens, int64_t requests, int kv_heads, int group, int D, int max_nodes, int window, int64_t width) {
  TreeShape s;
  const int64_t nodes = max_nodes < tokens ? max_nodes : tokens, rows = nodes * group;  // rows of a request and head, at most
  int64_t most = width;  // pages of a unit
  if (window > 0 && ((int64_t)window + nodes) / KV_PAGE + 2 < most) most = ((int64_t)window + nodes) / KV_PAGE + 2;
  // 8 kv heads of 128, us.  16 rows and fewer: the kernel of decoding (32 requests of 4000 30, here 40).  Little work: that one up to
  // 64 rows, as its first page takes fewer trips (32 rows: one request of 8000 17, here 23; 32 of 1500 25 and 31; 64 rows of one of
  // 8000 21 and 28), this one beyond (128 rows: one of 500 19 in the kernel of chunks and here 13, of 8000 35 and 31).  Otherwise
  // this one up to 96 rows (32: 16 of 16 000 98 and 82; 64: the same 168 and 117; 96: 32 of 4000 106 and 81), the
  // kernels of chunks beyond (128: 32 of 4000 113 and 129; 256: 152 and 222), but where requests have fewer tokens than the largest,
  // whose tiles they leave part empty (64 of up to 8000, trees of up to 128 rows 147 and 101, 512 365 and 286).
  const bool little = ((tokens * group + 15) / 16 + requests) * kv_heads * most < 32768;
  const bool ragged = tokens * 8 <= requests * nodes * 7;
  s.tiles = rows <= 16 ? 0 : little ? (rows > 64 ? NT : 0) : rows <= 96 || (ragged && rows <= 512) ? NT : 0;
  if (s.tiles == 0) {
    static_cast<Shape &>(s) = shape_of(tokens, requests, kv_heads, group, D, max_nodes, window, 0, width);
    return s;
  }
  const bool narrow = most <= WHOLE_PAGES;
  s.tile_rows = 16 * s.tiles;
  const int64_t units = s.units = (tokens * group / s.tile_rows + requests) * kv_heads;
  const int fill = D <= 128 ? 768 : 256;
  const int64_t surely = window > 0 ? (window + tokens) / KV_PAGE + 2 : width;
  s.whole = narrow || units * ((surely < width ? surely : width) + UNIT_EXTRA) > 0x7fffffff;
  const int shares = units * most / 4 >= fill ? fill : (int)(units * most / 4 + 1);
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
  a.scanned = a.requests > SCAN_REQUESTS;
  if (a.scanned) {
    hipLaunchKernelGGL(kv_scan_kernel, dim3(1), dim3(1024), 0, s, a, sh.tile_rows);
    KV_HIP_TRY(hipGetLastError());
  }
  const size_t lists = a.scanned ? 0 : ((size_t)a.requests + 3 * (size_t)(a.requests + 1)) * 4;
  const size_t lds = 8 * (size_t)half_bytes<D>() + sizeof(RowsInLds<D>) + 4 * 16 * 2 * 4 + 4 * 4 + lists;
  int rc;
  if ((rc = allow_lds(&kv_tiles_kernel<D, DT>, lds))) return rc;
  hipLaunchKernelGGL((kv_tiles_kernel<D, DT>), dim3((unsigned)a.n_wg), dim3(256), lds, s, a);
  KV_HIP_TRY(hipGetLastError());
  if (a.whole || a.n_wg == 1) return IVFPQ_OK;
  const int64_t most = a.tokens * (int64_t)a.group;
  const int rows = (int)(most < sh.tile_rows ? most : sh.tile_rows);
  // few units of dozens of parts each: a workgroup a row; many of two or three: a workgroup 256 / (D / 4) rows (800 units
  // over 768 shares: 21 us and 7)
  if (sh.n_wg >= 8 * sh.units) {
    hipLaunchKernelGGL((kv_join_kernel<D, DT, true>), dim3((unsigned)(a.n_wg - 1), (unsigned)rows), dim3(256), 0, s, a, sh.tile_rows);
  } else {
    constexpr int SETS = 256 / (D / 4);
    hipLaunchKernelGGL((kv_join_kernel<D, DT, false>), dim3((unsigned)(a.n_wg - 1), (unsigned)((rows + SETS - 1) / SETS)), dim3(256), 0, s, a,
                       sh.tile_rows);
  }
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

template <int D, int DT>
int tree_attention_of(const KvAttnArgs &a, const TreeShape &sh, hipStream_t s) {
  if (sh.tiles == 0) return attention_of<D, DT, true>(a, sh, s);
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

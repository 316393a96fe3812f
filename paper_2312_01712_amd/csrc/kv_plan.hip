// Page tables and slot maps of a step from the requests' lengths, on the device: a server that
// builds them on the host has to bring the lengths back first.
//
// Workgroup (b, part) owns per_group requests; it sums what all requests before them
// add, take and give back, scans its own, and writes their part of
// the slots, the table and the ring.  Nothing is written that another workgroup reads: the new
// counters go to an array of their own, pages are taken from [head, tail) of the ring and given
// back behind tail, entries of the table are read below ceil(past / 64) and written from there.
//
// An ended request gives back the pages that it has, not the columns that its length covers: where
// pages ran out its row has -1, and those in the ring would let it claim more pages than there are.
// So its row is counted before anything is placed: with few requests by every workgroup, for the requests up to its own;
// otherwise by a launch of its own, which leaves sums of 16 requests too, so that no workgroup reads all lengths.
// Bound by the launch and a few dependent trips to L2: 4.2 us for one request of 37 tokens, 3.8 and 9.1 us for 4001 requests
// (15 000 new tokens, 250 of them ended with up to 2046 pages each).

#include "kv_internal.h"

namespace ivfpq {

namespace {

// held: pages that its length covers; take: pages that it needs beyond them
struct Counts {
  int32_t past, fresh, held, take;
};

// a request's lengths, cut to what its row of the table has room for
__device__ inline Counts counts_of(int32_t past, int32_t fresh, int32_t width) {
  Counts c;
  const int64_t room = (int64_t)width * KV_PAGE;
  c.past = past < 0 ? 0 : (int32_t)(past < room ? past : room);
  c.fresh = fresh < 0 ? 0 : fresh;
  c.held = (int32_t)(((int64_t)c.past + KV_PAGE - 1) / KV_PAGE);
  int64_t total = (int64_t)c.past + c.fresh;
  total = total < room ? total : room;
  c.take = fresh < 0 ? 0 : (int32_t)((total + KV_PAGE - 1) / KV_PAGE) - c.held;
  return c;
}

__device__ inline int64_t wave_sum(int64_t v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Pages among the first n entries of a row, by a wavefront: sixteen loads a lane on their way at a time.
__device__ inline int32_t count_pages(const int32_t *row, int32_t n, int lane) {
  int32_t pages = 0;
  for (int b = 0; b < n; b += 16 * 64) {
    int32_t page[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) page[k] = row[min(b + k * 64 + lane, n - 1)];
#pragma unroll
    for (int k = 0; k < 16; ++k) pages += b + k * 64 + lane < n && page[k] >= 0;
  }
  for (int d = 32; d > 0; d >>= 1) pages += __shfl_xor(pages, d);
  return pages;
}

constexpr int PLAN_PER_GROUP = 16;  // most requests that a workgroup owns
constexpr int WIDE = 256;           // pages given back by more than one wavefront
constexpr int COUNT_HERE = 8;       // requests below which every workgroup counts the pages of ended ones itself

// Pages that the ended requests have, a wavefront a row; a workgroup has 16 requests and leaves what they add, take and give, or,
// where no totals are wanted, four.
__global__ __launch_bounds__(256) void kv_count_kernel(KvPlanArgs a) {
  __shared__ int32_t give[PLAN_PER_GROUP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = a.totals ? PLAN_PER_GROUP : 4, r0 = blockIdx.x * per;
  const int r = min(r0 + (lane & 15), a.requests - 1);
  const bool own = lane < per && r0 + lane < a.requests;
  const int32_t fresh = a.fresh[r];
  const Counts c = counts_of(a.past[r], fresh, a.width);
  if (threadIdx.x < PLAN_PER_GROUP) give[threadIdx.x] = 0;
  __syncthreads();
  int k = 0;
  for (uint64_t todo = __ballot(own && fresh < 0); todo; todo &= todo - 1, ++k) {
    if ((k & 3) != wave) continue;
    const int j = __builtin_ctzll(todo);
    const int32_t pages = count_pages(a.table + (int64_t)(r0 + j) * a.width, __shfl(c.held, j), lane);
    if (lane == 0) give[j] = a.counts[r0 + j] = pages;
  }
  __syncthreads();
  if (wave > 0 || !a.totals) return;
  // (new tokens beyond the step's rows are the same whatever their number, and 16 requests' stay in 32 bits)
  int32_t t0 = own ? min(c.fresh, a.max_tokens + 1) : 0, t1 = own ? c.take : 0, t2 = own ? give[lane] : 0;
  for (int d = 8; d > 0; d >>= 1) t0 += __shfl_xor(t0, d), t1 += __shfl_xor(t1, d), t2 += __shfl_xor(t2, d);
  if (lane == 0) {
    int32_t *to = a.totals + blockIdx.x * 3;
    to[0] = t0, to[1] = t1, to[2] = t2;
  }
}

__global__ __launch_bounds__(256) void kv_plan_kernel(KvPlanArgs a) {
  __shared__ int64_t before[3], sums[4][3];
  __shared__ int32_t own[PLAN_PER_GROUP][6];  // first token, first page taken, first page given, past, fresh, pages given
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r0 = blockIdx.x * a.per_group, part = blockIdx.y;
  const int n_own = min(a.per_group, a.requests - r0);

  // eight requests a thread in flight: their lengths are in L2 and what counts is the trip to it
  int64_t s0 = 0, s1 = 0, s2 = 0;
  if (!a.counts) {
    // the ended requests up to the own ones, a wavefront's lanes look 64 of them up at a time
    for (int b = wave * 64; b < r0 + n_own; b += 256) {
      const int r = min(b + lane, r0 + n_own - 1);
      const Counts c = counts_of(a.past[r], a.fresh[r], a.width);
      for (uint64_t todo = __ballot(b + lane < r0 + n_own && a.fresh[r] < 0); todo; todo &= todo - 1) {
        const int j = __builtin_ctzll(todo), ended = b + j;
        const int32_t pages = count_pages(a.table + (int64_t)ended * a.width, __shfl(c.held, j), lane);
        if (lane == 0 && ended < r0) s2 += pages;
        if (lane == 0 && ended >= r0) own[ended - r0][5] = pages;
      }
    }
  }
  if (a.totals)
    for (int g = tid; g < (int)blockIdx.x; g += 256) s0 += a.totals[g * 3], s1 += a.totals[g * 3 + 1], s2 += a.totals[g * 3 + 2];
  for (int b = 0; b < (a.totals ? 0 : r0); b += 8 * 256) {
    int32_t past[8], fresh[8], pages[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int r = min(b + k * 256 + tid, r0);  // (request r0 exists)
      past[k] = a.past[r];
      fresh[k] = a.fresh[r];
      pages[k] = a.counts ? a.counts[r] : 0;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (b + k * 256 + tid < r0) {
        const Counts c = counts_of(past[k], fresh[k], a.width);
        s0 += c.fresh;
        s1 += c.take;
        s2 += fresh[k] < 0 ? pages[k] : 0;
      }
  }
  s0 = wave_sum(s0);
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if (lane == 0) sums[wave][0] = s0, sums[wave][1] = s1, sums[wave][2] = s2;
  __syncthreads();
  if (wave == 0) {
    // own requests, a lane each, scanned behind the sums
    Counts c = {0, 0, 0, 0};
    int32_t fresh_raw = 0, give = 0;
    if (lane < n_own) {
      fresh_raw = a.fresh[r0 + lane];
      c = counts_of(a.past[r0 + lane], fresh_raw, a.width);
      if (fresh_raw < 0) give = a.counts ? a.counts[r0 + lane] : own[lane][5];
    }
    int64_t t0 = c.fresh, t1 = c.take, t2 = give;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t u0 = __shfl_up(t0, d), u1 = __shfl_up(t1, d), u2 = __shfl_up(t2, d);
      if (lane >= d) t0 += u0, t1 += u1, t2 += u2;
    }
    for (int w = 0; w < 4; ++w) t0 += sums[w][0], t1 += sums[w][1], t2 += sums[w][2];
    if (lane < n_own) {
      own[lane][0] = (int32_t)min(t0 - c.fresh, (int64_t)a.max_tokens);
      own[lane][1] = (int32_t)min(t1 - c.take, (int64_t)0x7fffffff);
      own[lane][2] = (int32_t)min(t2 - give, (int64_t)0x7fffffff);
      own[lane][3] = c.past;
      own[lane][4] = fresh_raw;
      own[lane][5] = give;
      if (part == 0) {
        const int64_t room = (int64_t)a.width * KV_PAGE, total = (int64_t)c.past + c.fresh;
        a.kv_lens[r0 + lane] = fresh_raw < 0 ? 0 : (int32_t)(total < room ? total : room);
        a.q_start[r0 + lane] = own[lane][0];
      }
    }
    if (lane == 63) before[0] = t0, before[1] = t1, before[2] = t2;
  }
  __syncthreads();

  const int64_t head = a.state[0], tail = a.state[1];
  const int64_t avail = tail > head ? min(tail - head, a.capacity) : 0;
  const int64_t room = a.capacity - avail;  // no page is put onto one that waits in the ring
  const int32_t cap = (int32_t)a.capacity;
  int32_t head_at = (int32_t)(head % a.capacity), tail_at = (int32_t)(tail % a.capacity);
  if (head_at < 0) head_at += cap;  // counters that were never set up: still inside the ring
  if (tail_at < 0) tail_at += cap;
  const bool last = r0 + n_own == a.requests;
  if (last && part == 0 && tid == 0) {
    const int64_t used = min(before[1], avail);
    a.state_out[0] = head + used;
    a.state_out[1] = tail + min(before[2], room);
    a.state_out[2] = before[1] - used;
    a.q_start[a.requests] = (int32_t)min(before[0], (int64_t)a.max_tokens);
  }

  // page `to` of all that are given back
  auto put = [&](int64_t to, int32_t page) {
    if (to >= room) return;
    int64_t at = tail_at + to;
    if (at >= cap) at -= cap;
    a.free_pages[at] = page;
  };
  // the columns of an ended request, all of them pages, from `first` on every `stride`-th: eight loads on their way at a time
  auto give_back = [&](const int32_t *row, int32_t before_it, int32_t n, int first, int stride) {
    for (int b = first; b < n; b += 8 * stride) {
      int32_t page[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) page[k] = row[min(b + k * stride, n - 1)];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (b + k * stride < n) put((int64_t)before_it + b + k * stride, page[k]);
    }
  };
  // those of a request that lacked pages, by a wavefront
  auto give_back_some = [&](const int32_t *row, int32_t before_it, int32_t n) {
    int64_t to = before_it;
    for (int b = 0; b < n; b += 64) {
      const int32_t page = b + lane < n ? row[b + lane] : -1;
      const uint64_t there = __ballot(page >= 0);
      if (page >= 0) put(to + __builtin_popcountll(there & ((1ull << lane) - 1)), page);
      to += __builtin_popcountll(there);
    }
  };
  // many pages: the whole workgroup on a request
  if (a.parts == 1)
    for (int i = 0; i < n_own; ++i) {
      const int32_t give = own[i][5];
      if (give > WIDE && give == counts_of(own[i][3], own[i][4], a.width).held)
        give_back(a.table + (int64_t)(r0 + i) * a.width, own[i][2], give, tid, 256);
    }

  const int n_waves = 4 * a.parts, w = part * 4 + wave;  // all of them on one request after the other when there are few
  for (int i = a.parts == 1 ? wave : 0; i < n_own; i += a.parts == 1 ? 4 : 1) {
    const int r = r0 + i, first = a.parts == 1 ? lane : w * 64 + lane, stride = a.parts == 1 ? 64 : n_waves * 64;
    const int32_t past = own[i][3], fresh = own[i][4];
    const Counts c = counts_of(past, fresh, a.width);
    int32_t *row = a.table + (int64_t)r * a.width;
    // page `take` of this request, or -1
    auto taken = [&](int32_t j) -> int32_t {
      const int64_t n = (int64_t)own[i][1] + j;
      if (n >= avail) return -1;
      int64_t at = head_at + n;
      if (at >= cap) at -= cap;
      return a.free_pages[at];
    };
    const int32_t give = own[i][5];
    if (give > 0 && give < c.held) {
      if (a.parts == 1 || w == 0) give_back_some(row, own[i][2], c.held);
    } else if (give <= WIDE || a.parts > 1) {
      give_back(row, own[i][2], give, first, stride);
    }
    for (int j = first; j < c.take; j += stride) row[c.held + j] = taken(j);
    for (int64_t j = first; j < c.fresh; j += stride) {
      const int64_t t = own[i][0] + j, pos = c.past + j;
      if (t >= a.max_tokens) break;
      const int64_t col = pos / KV_PAGE;
      int32_t page = -1;
      if (col < c.held) page = row[col];
      else if (col < c.held + c.take) page = taken((int32_t)(col - c.held));
      a.slots[t] = page >= 0 ? (int64_t)page * KV_PAGE + pos % KV_PAGE : -1;
      a.token_req[t] = r;
      a.positions[t] = (int32_t)pos;
    }
  }
  if (last)  // rows that stand for no token
    for (int64_t t = before[0] + part * 256 + tid; t < a.max_tokens; t += (int64_t)a.parts * 256) {
      a.slots[t] = -1;
      a.token_req[t] = -1;
      a.positions[t] = -1;
    }
}

}  // namespace

int launch_kv_plan(const KvPlanArgs &args, hipStream_t s) {
  KvPlanArgs a = args;
  // a wavefront for each request when there are many; all of a part's wavefronts on one request
  // after the other when there are few and each may have many tokens
  a.per_group = a.requests >= 64 ? PLAN_PER_GROUP : 1;
  const int64_t groups = a.requests > 0 ? (a.requests + a.per_group - 1) / a.per_group : 1;
  int64_t parts = 1;
  if (a.requests < 64) {
    const int64_t want = ((int64_t)a.max_tokens + 1023) / 1024, most = 512 / groups;
    parts = want < 1 ? 1 : want > most ? most : want;
  }
  a.parts = (int32_t)parts;
  // Ended requests' pages: counted here in one launch, there in two (8 requests of 130 000 tokens, half of them ended: 10.2 and
  // 9.5 us, 15: 13.7 and 9.5).
  if (a.requests < COUNT_HERE) a.counts = nullptr;
  a.totals = a.counts && a.per_group == PLAN_PER_GROUP ? a.counts + a.requests : nullptr;
  if (a.counts) {
    hipLaunchKernelGGL(kv_count_kernel, dim3((unsigned)(a.totals ? groups : (a.requests + 3) / 4)), dim3(256), 0, s, a);
    KV_HIP_TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(kv_plan_kernel, dim3((unsigned)groups, (unsigned)parts), dim3(256), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

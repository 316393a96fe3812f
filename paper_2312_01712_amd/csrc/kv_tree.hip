// Trees of drafted tokens: what each sees of the others and its position, from the tokens' parents; and the tokens of a
// tree that stay, from what the model picked behind each.

#include "kv_internal.h"

namespace ivfpq {

namespace {

// A request's new tokens: first row and number, both inside the step's rows.
struct Fresh {
  int t0, n;
};

__device__ inline Fresh fresh_of(const int32_t *q_start, int r, int tokens) {
  const int t0 = min(max(q_start[r], 0), tokens);
  return {t0, max(min(q_start[r + 1], tokens) - t0, 0)};
}

// Workgroup (r, y): words WORDS y .. of the masks of request r's tokens, a thread a token.  Ancestors by doubling: after k turns a thread
// has the set of its token and the 2^k - 1 ancestors next to it, and the 2^k-th ancestor; the next turn adds that one's set.  As
// many turns as the depth has bits.  A window takes the sets of its size's bits, one behind the other.  Bound by the launch and
// the trips lengths - parents: 5.6 us for 700 requests of up to 200 tokens (a word a workgroup: 8.3), 2.2 for one of 26.
template <int THREADS, int WORDS>
__global__ __launch_bounds__(THREADS) void kv_tree_kernel(KvTreeArgs a) {
  __shared__ uint64_t set[WORDS][THREADS];
  __shared__ int32_t up[THREADS], far[THREADS];
  const int i = threadIdx.x, r = blockIdx.x, w0 = blockIdx.y * WORDS;
  if (r < a.requests) {
    const Fresh f = fresh_of(a.q_start, r, a.tokens);
    const int n = min(f.n, a.max_nodes);
    const bool windowed = a.window > 0 && a.window < n;
    int parent = -1;
    if (i < n) {
      const int p = a.parents[f.t0 + i];
      if (p >= 0 && p < i) parent = p;
    }
    const int first = f.n > 0 ? a.positions[f.t0] : 0;
    uint64_t mine[WORDS], sees[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      mine[w] = (i >> 6) == w0 + w ? 1ull << (i & 63) : 0;
      sees[w] = 0;
    }
    int steps = parent >= 0, at = i;
    for (int k = 0; (1 << k) < n; ++k) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w) set[w][i] = mine[w];
      up[i] = parent;
      far[i] = steps;
      const bool more = __syncthreads_or(parent >= 0);
      if (windowed && (a.window >> k & 1) && at >= 0) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) sees[w] |= set[w][at];
        at = up[at];
      }
      if (!more && !windowed) break;
      if (parent >= 0) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) mine[w] |= set[w][parent];
        steps += far[parent];
        parent = up[parent];
      }
      __syncthreads();
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      if (w0 + w >= a.words) break;
      if (i < n) a.masks[(int64_t)(f.t0 + i) * a.words + w0 + w] = windowed ? sees[w] : mine[w];
      // tokens that the masks have no room for
      for (int j = a.max_nodes + i; j < f.n; j += THREADS) a.masks[(int64_t)(f.t0 + j) * a.words + w0 + w] = 0;
    }
    if (w0 == 0) {
      if (i < n) a.tree_positions[f.t0 + i] = first + steps;
      for (int j = a.max_nodes + i; j < f.n; j += THREADS) a.tree_positions[f.t0 + j] = -1;
    }
  }
  // rows that stand for no token
  const int end = a.requests > 0 ? min(max(a.q_start[a.requests], 0), a.tokens) : 0;
  for (int64_t t = end + (int64_t)r * THREADS + i; t < a.tokens; t += (int64_t)gridDim.x * THREADS) {
    for (int w = w0; w < min(w0 + WORDS, a.words); ++w) a.masks[t * a.words + w] = 0;
    if (w0 == 0) a.tree_positions[t] = -1;
  }
}

// Workgroup r: request r's path.  A token agrees if it is the first of its request, or is what was picked behind its parent (its
// last ancestor: the highest bit below its own); it can stay if all that it sees agree.  The deepest of these, the first
// among equals, and what it sees stay.  Bound by the launch and its trips: 2.7 us for one request, 4.1 for 48.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_accept_kernel(KvKeepArgs a) {
  __shared__ uint64_t agree[THREADS / 64], path[THREADS / 64];
  __shared__ int best[THREADS / 64];
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6, r = blockIdx.x;
  if (r < a.requests) {
    const Fresh f = fresh_of(a.q_start, r, a.tokens);
    const int n = min(f.n, a.max_nodes), words = a.words, kv = a.kv_lens[r];
    const uint64_t *mask = a.masks + (int64_t)(f.t0 + i) * words;
    auto named = [&](int w) -> uint64_t {  // without bits of tokens that are not there
      const int there = n - w * 64;
      return mask[w] & (there >= 64 ? ~0ull : there > 0 ? (1ull << there) - 1 : 0);
    };
    bool agrees = false;
    if (i < n) {
      const int64_t slot = a.slots[f.t0 + i];
      if (i == 0) {
        agrees = true;
      } else if (slot >= 0 && slot < a.n_pages * KV_PAGE) {
        int w = i >> 6;
        uint64_t below = mask[w] & ((1ull << (i & 63)) - 1);
        while (below == 0 && w > 0) below = mask[--w];
        if (below != 0) {
          const int parent = w * 64 + 63 - __builtin_clzll(below);
          agrees = a.drafted[f.t0 + i] == a.picked[f.t0 + parent];
        }
      }
    }
    const uint64_t vote = __ballot(agrees);
    if (lane == 0) agree[wave] = vote, path[wave] = 0;
    __syncthreads();
    int rank = -1;
    if (i < n) {
      bool good = true;
      int depth = 0;
      for (int w = 0; w < words; ++w) {
        const uint64_t x = named(w);
        good = good && (x & ~agree[w]) == 0;
        depth += __builtin_popcountll(x);
      }
      if (good) rank = depth * 1024 + 1023 - i;
    }
    int top = rank;
    for (int d = 32; d > 0; d >>= 1) top = max(top, __shfl_xor(top, d));
    if (lane == 0) best[wave] = top;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, best[w]);
    if (rank >= 0 && rank == top)
      for (int w = 0; w < words; ++w) path[w] = named(w);
    __syncthreads();
    int kept = 0, before = 0;
    for (int w = 0; w < words; ++w) {
      if (w < wave) before += __builtin_popcountll(path[w]);
      kept += __builtin_popcountll(path[w]);
    }
    if (i < n && (path[wave] >> lane & 1)) a.rows[f.t0 + before + __builtin_popcountll(path[wave] & ((1ull << lane) - 1))] = f.t0 + i;
    for (int j = kept + i; j < f.n; j += THREADS) a.rows[f.t0 + j] = -1;
    // what is held from now on, and how many pages lie behind it
    const int stays = f.n > 0 ? min(max(a.positions[f.t0], 0) + kept, kv) : kv;
    if (wave == 0) {
      const int from = (int)(((int64_t)stays + KV_PAGE - 1) / KV_PAGE), to = min((int)(((int64_t)kv + KV_PAGE - 1) / KV_PAGE), a.width);
      int back = 0;
      for (int c = from; c < to; c += 64) {
        const int page = c + lane < to ? a.table[(int64_t)r * a.width + c + lane] : -1;
        back += __builtin_popcountll(__ballot((uint32_t)page < (uint64_t)a.n_pages));
      }
      if (lane == 0) a.lens[r] = stays, a.counts[r] = back;
    }
  }
  const int end = a.requests > 0 ? min(max(a.q_start[a.requests], 0), a.tokens) : 0;
  for (int64_t t = end + (int64_t)r * THREADS + i; t < a.tokens; t += (int64_t)gridDim.x * THREADS) a.rows[t] = -1;
}

}  // namespace

int launch_kv_tree(const KvTreeArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(a.requests > 0 ? a.requests : 1), (unsigned)((a.words + 3) / 4));
  if (a.max_nodes <= 64) hipLaunchKernelGGL((kv_tree_kernel<64, 1>), grid, dim3(64), 0, s, a);
  else if (a.max_nodes <= 256) hipLaunchKernelGGL((kv_tree_kernel<256, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_tree_kernel<1024, 4>), grid, dim3(1024), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

int launch_kv_accept(const KvKeepArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(a.requests > 0 ? a.requests : 1));
  if (a.max_nodes <= 64) hipLaunchKernelGGL((kv_accept_kernel<64>), grid, dim3(64), 0, s, a);
  else if (a.max_nodes <= 256) hipLaunchKernelGGL((kv_accept_kernel<256>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_accept_kernel<1024>), grid, dim3(1024), 0, s, a);
  KV_HIP_TRY(hipGetLastError());
  return IVFPQ_OK;
}

}  // namespace ivfpq

// Page tables of a step, from the lengths held and the lengths to come: pages given back and taken, the new tokens' offsets in
// the packed batch, their positions and their slots.
//
// Whole numbers and latency: every CTA scans the sequences (new tokens, pages given back, pages wanted) into shared memory and
// then takes its part of three flat lists, finding an entry's sequence by bisection: the pages given back (onto the stack of
// free ones), the pages taken (from its top, those just given back included, so an entry may come straight from a table row),
// and the new tokens, four at a time.  The stack's live entries and the tables' live entries are only read and what is written
// lies behind them, so nothing has to wait; the two counters that may be updated in place are written by the last CTA to finish.
// 64 sequences' step 5.1 us, 128 new prompts of up to 2048 rows 5.8, 512 sequences of which some grow, end or are cut 10.5.
#include <algorithm>

#include "chunk_step.cuh"

namespace earn {
namespace {

__device__ __forceinline__ int pages_of(int rows) { return (rows + EARN_PAGE_TOKENS - 1) / EARN_PAGE_TOKENS; }

// last index i < n with from[i] <= x (from[0] = 0, increasing): the sequence that entry x belongs to
__device__ __forceinline__ int find(const int* from, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (from[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Inclusive sums of two numbers over the block's threads, and their totals.  `warps`: shared memory for 32 pairs, another one
// than the last call's.
template <int THREADS, typename A>
__device__ __forceinline__ void block_scan(A& a, int& b, A& all_a, int& all_b, A* warps_a, int* warps_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const A u = __shfl_up_sync(0xffffffffu, a, d);
    const int v = __shfl_up_sync(0xffffffffu, b, d);
    if (lane >= d) { a += u; b += v; }
  }
  if (lane == 31) { warps_a[warp] = a; warps_b[warp] = b; }
  __syncthreads();
  A x = lane < THREADS / 32 ? warps_a[lane] : 0;
  int y = lane < THREADS / 32 ? warps_b[lane] : 0;
#pragma unroll
  for (int d = 1; d < THREADS / 32; d <<= 1) {
    const A u = __shfl_up_sync(0xffffffffu, x, d);
    const int v = __shfl_up_sync(0xffffffffu, y, d);
    if (lane >= d) { x += u; y += v; }
  }
  all_a = __shfl_sync(0xffffffffu, x, THREADS / 32 - 1);
  all_b = __shfl_sync(0xffffffffu, y, THREADS / 32 - 1);
  const A before_a = __shfl_sync(0xffffffffu, x, warp > 0 ? warp - 1 : 0);
  const int before_b = __shfl_sync(0xffffffffu, y, warp > 0 ? warp - 1 : 0);
  if (warp > 0) { a += before_a; b += before_b; }
}

struct Want {
  int held, target;   // target >= 0; may lie past the table
};
__device__ __forceinline__ Want want_of(const PageTableArgs& a, int b) {
  Want w;
  w.held = min(max(a.held[b], 0), a.pages_per_seq * EARN_PAGE_TOKENS);
  w.target = max(a.target[b], 0);
  return w;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) page_tables_kernel(PageTableArgs a) {
  extern __shared__ int from[];            // three lists of n_seq: first token, first page taken, first page given back
  int* tok_from = from;
  int* take_from = from + a.n_seq;         // bit 31: the sequence is refused
  int* back_from = take_from + a.n_seq;
  __shared__ int64_t warps_a[2][32];
  __shared__ int warps_b[4][32], last;
  const int t = threadIdx.x, cap = a.pages_per_seq * EARN_PAGE_TOKENS;
  pdl_launch_dependents();
  pdl_wait();
  const int n_free = min(max(*a.n_free, 0), a.n_pages);
  // ---- tokens and pages given back
  int64_t tokens = 0;
  int back = 0, turn = 0;   // (pages given back: at most as many as there are rows of tables, and no more are used than n_pages)
  for (int b0 = 0; b0 < a.n_seq; b0 += THREADS, turn ^= 1) {
    const int b = b0 + t;
    int grow = 0, give = 0;
    Want w{0, 0};
    if (b < a.n_seq) {
      w = want_of(a, b);
      grow = max(w.target - w.held, 0);
      give = max(pages_of(w.held) - pages_of(min(w.target, cap)), 0);
    }
    int64_t tok = grow, sum_tok;
    int bk = min(give, a.n_pages), sum_back;
    block_scan<THREADS>(tok, bk, sum_tok, sum_back, warps_a[turn], warps_b[turn]);
    tok += tokens;
    bk = max(min(bk + back, a.n_pages), 0);
    if (b < a.n_seq) {
      tok_from[b] = (int)min(tok - grow, (int64_t)a.n_tokens);
      back_from[b] = max(bk - give, 0);
      take_from[b] = grow == 0 || (tok <= a.n_tokens && w.target <= cap) ? max(pages_of(min(w.target, cap)) - pages_of(w.held), 0) : -1;
    }
    tokens += sum_tok;
    back = max(min(back + sum_back, a.n_pages), 0);
  }
  const int room = min(n_free + back, a.n_pages);
  // ---- pages wanted, first come first served
  int64_t wanted = 0;
  int n_taken = 0, n_refused = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += THREADS, turn ^= 1) {
    const int b = b0 + t, need = b < a.n_seq ? take_from[b] : 0;
    int64_t end = max(need, 0), sum;
    int refused = need < 0 ? 1 : 0, sum_refused;
    block_scan<THREADS>(end, refused, sum, sum_refused, warps_a[turn], warps_b[2 + turn]);
    end += wanted;
    const bool ok = need == 0 || (need > 0 && end <= room);
    if (b < a.n_seq) take_from[b] = (int)min(end - max(need, 0), (int64_t)a.n_pages) | (ok ? 0 : (int)0x80000000);
    // granted ones come before the first one that there are no pages for: the last of them tells how many pages are taken
    n_taken = max(n_taken, __reduce_max_sync(0xffffffffu, ok && need > 0 ? (int)end : 0));
    n_refused += __popc(__ballot_sync(0xffffffffu, b < a.n_seq && !ok));
    wanted += sum;
  }
  if ((t & 31) == 0) { warps_b[turn][t >> 5] = n_taken; warps_b[2 + turn][t >> 5] = n_refused; }
  __syncthreads();
  n_taken = __reduce_max_sync(0xffffffffu, (t & 31) < THREADS / 32 ? warps_b[turn][t & 31] : 0);
  n_refused = __reduce_add_sync(0xffffffffu, (t & 31) < THREADS / 32 ? warps_b[2 + turn][t & 31] : 0);
  const int n_back = room - n_free, at = blockIdx.x * THREADS + t, step = gridDim.x * THREADS;
  // entry `i` of the stack of free pages, once all pages given back lie on it
  auto stack = [&](int i) {
    if (i < n_free) return a.free_pages[i];
    const int b = find(back_from, a.n_seq, i - n_free);
    const int p = pages_of(min(max(a.target[b], 0), cap)) + (i - n_free - back_from[b]);   // (in the row unless the pool is broken)
    return a.block_table[(int64_t)b * a.pages_per_seq + min(max(p, 0), a.pages_per_seq - 1)];
  };
  // the list of pages taken has refused sequences in it, all of them behind the last page taken
  auto take_first = [&](int b) { return take_from[b] & 0x7fffffff; };
  for (int i = at; i < n_back; i += step) a.free_pages[n_free + i] = stack(n_free + i);
  for (int i = at; i < n_taken; i += step) {
    int lo = 0, hi = a.n_seq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (take_first(mid) <= i) lo = mid; else hi = mid;
    }
    const int p = pages_of(min(max(a.held[lo], 0), cap)) + (i - take_first(lo));
    if (p < a.pages_per_seq) a.block_table[(int64_t)lo * a.pages_per_seq + p] = stack(room - 1 - i);
  }
  // ---- positions and slots
  const int live = (int)min(tokens, (int64_t)a.n_tokens);
  for (int j0 = at * 4; j0 < a.n_tokens; j0 += step * 4) {
    int pos[4], slot[4];
    int b = j0 < live ? find(tok_from, a.n_seq, j0) : 0, page_at = -1, page = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + e;
      pos[e] = slot[e] = -1;
      if (j >= live) continue;
      while (b + 1 < a.n_seq && tok_from[b + 1] <= j) { ++b; page_at = -1; }
      if (take_from[b] < 0) continue;
      const int held = min(max(a.held[b], 0), cap);
      pos[e] = held + j - tok_from[b];
      const int p = pos[e] / EARN_PAGE_TOKENS;
      if (p != page_at) {
        const int have = pages_of(held);
        page = p < have ? a.block_table[(int64_t)b * a.pages_per_seq + p] : stack(room - 1 - take_first(b) - (p - have));
        page_at = p;
      }
      slot[e] = page * EARN_PAGE_TOKENS + pos[e] % EARN_PAGE_TOKENS;
    }
    if (j0 + 4 <= a.n_tokens) {
      *reinterpret_cast<int4*>(a.positions + j0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(a.slots + j0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
      for (int e = 0; j0 + e < a.n_tokens; ++e) { a.positions[j0 + e] = pos[e]; a.slots[j0 + e] = slot[e]; }
    }
  }
  // ---- what is written once
  if (blockIdx.x == 0) {
    for (int b = t; b < a.n_seq; b += THREADS) {
      a.cu_new[b] = tok_from[b];
      a.seq_len[b] = take_from[b] < 0 ? 0 : max(a.target[b], 0);
    }
    if (t == 0) {
      a.cu_new[a.n_seq] = live;
      *a.n_refused = n_refused;
    }
  }
  __syncthreads();   // (reads of held and n_free by this CTA are over)
  if (gridDim.x > 1) {
    if (t == 0) {
      __threadfence();
      last = last_arrival(a.ticket, (int)gridDim.x, a.status);
      __threadfence();
    }
    __syncthreads();
    if (!last) return;
  }
  for (int b = t; b < a.n_seq; b += THREADS) {
    const Want w = want_of(a, b);
    a.held_out[b] = take_from[b] < 0 ? w.held : w.target;
  }
  if (t == 0) *a.n_free_out = room - n_taken;
}

}  // namespace

template <int THREADS>
static cudaError_t launch(const PageTableArgs& a, cudaStream_t st) {
  const int bytes = 3 * 4 * a.n_seq;
  // a thread has four tokens: one CTA for a step's worth, more for prompts, each with the scan of the sequences before it
  const int grid = std::max(1, std::min(sm_count(), (a.n_tokens + 4 * THREADS - 1) / (4 * THREADS)));
  cudaError_t e = bytes > 32768 ? ensure_dynamic_smem<page_tables_kernel<THREADS>>(3 * 4 * kPageTablesMaxSeqs) : cudaSuccess;
  if (e == cudaSuccess) e = launch_pdl(page_tables_kernel<THREADS>, dim3(grid), dim3(THREADS), bytes, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

// Few threads have fewer warps to scan and to wait for, and more CTAs share the tokens: 512 sequences of a mixed step take 10.6 us
// with 512 threads, 10.5 with 256, 12.5 with 1024; 1000 of them 12.3, 13.7 and 13.9.
cudaError_t launch_page_tables(const PageTableArgs& a, cudaStream_t st) {
  return a.n_seq <= 256 ? launch<256>(a, st) : a.n_seq <= 1024 ? launch<512>(a, st) : launch<1024>(a, st);
}

}  // namespace earn

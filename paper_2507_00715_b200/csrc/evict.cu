// Eviction from a cache by accumulated attention weight: which rows of every (sequence, kv head) stay within the budget,
// and their way into (prompt form) or inside (step form) the paged cache.
//
// Selection: every row gets a 32-bit key that orders as the policy does (a protected row the largest key of all, otherwise
// the weight's bits made monotone), and the budget-th largest key is found digit by digit with a histogram in shared memory;
// of the rows that equal it the first ones stay.  Row numbers in order come from ballots: a warp owns a contiguous stretch of
// the list, so a count per warp turns into ranks.  Exact, and no result depends on the order in which threads arrive.
//   prompt form: the m-th kept position goes to pos_out[m], its K / V rows (bit copies, 16-byte vectors) from the packed
//   prompt into row m of the pages;
//   step form: the i-th free row below the budget and the i-th kept row behind it form a move; sources and destinations are
//   disjoint, so the moves run in any order.
// Lists of up to 65536 rows are selected by clusters (evict_cluster_kernel), which also copy unless the lists are more than
// one wave of them; longer lists by a kernel of one CTA each.  Where the selecting launch does not copy, a second one does.
// Times in this file are of calls replayed from a graph.
#include <climits>
#include <type_traits>

#include "paged_cache.cuh"

namespace earn {
namespace {

constexpr int DIGIT_BINS = 2048;

// monotone key of a weight: a larger key is a larger weight; -0 counts as 0 and NaN as -inf
__device__ __forceinline__ uint32_t weight_key(float w) {
  uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) u = 0xff800000u;
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
constexpr uint32_t KEY_PROTECTED = 0xffffffffu;

template <int NT>
__device__ __forceinline__ int2 block_exclusive_scan(int2 v, int2* warp_tot, int2& total) {   // warp_tot: NT / 32 + 1 entries
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int2 inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
    if (lane >= o) { inc.x += x; inc.y += y; }
  }
  __syncthreads();   // (the last scan's totals have been read)
  if (lane == 31) warp_tot[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    int2 t = lane < NT / 32 ? warp_tot[lane] : make_int2(0, 0);
    int2 ti = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, ti.x, o), y = __shfl_up_sync(0xffffffffu, ti.y, o);
      if (lane >= o) { ti.x += x; ti.y += y; }
    }
    if (lane < NT / 32) warp_tot[lane] = make_int2(ti.x - t.x, ti.y - t.y);
    if (lane == 31) warp_tot[NT / 32] = ti;
  }
  __syncthreads();
  total = warp_tot[NT / 32];
  const int2 base = warp_tot[warp];
  return make_int2(base.x + inc.x - v.x, base.y + inc.y - v.y);
}

struct SelectShared {
  int hist[DIGIT_BINS];
  int2 warp_tot[33];
  int bucket, rest, last;
};

// one head's K and V rows `from` -> `to` of sequence b (page rows), by `lanes` threads of which this is number `lane`
__device__ __forceinline__ void move_row(const EvictArgs& a, int b, int kvh, int from, int to, int lane, int lanes) {
  bool ok_from, ok_to;
  const int pf = paged_page(a.cache, b, from / EARN_PAGE_TOKENS, ok_from), pt = paged_page(a.cache, b, to / EARN_PAGE_TOKENS, ok_to);
  if (!ok_to) return;
  const int64_t src = (((int64_t)pf * EARN_PAGE_TOKENS + from % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes;
  const int64_t dst = (((int64_t)pt * EARN_PAGE_TOKENS + to % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes;
  for (int i = lane * 16; i < a.row_bytes; i += lanes * 16) {
    const uint4 x = *reinterpret_cast<const uint4*>(a.cache.k + src + i), y = *reinterpret_cast<const uint4*>(a.cache.v + src + i);
    *reinterpret_cast<uint4*>(a.cache.k + dst + i) = x;
    *reinterpret_cast<uint4*>(a.cache.v + dst + i) = y;
  }
}

// ---- lists of any length: one CTA per list, the keys read again from L2 for every step
constexpr int SELECT_THREADS = 1024;

template <bool PROMPT>
__global__ void __launch_bounds__(SELECT_THREADS) evict_select_kernel(EvictArgs a) {
  constexpr int NT = SELECT_THREADS;
  __shared__ SelectShared sh;
  pdl_wait();   // everything below reads or writes global memory
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, b = unit / a.Hkv, kvh = unit - b * a.Hkv;
  const int64_t cap = (int64_t)EARN_PAGE_TOKENS * a.cache.pages_per_seq;
  const int lo = PROMPT ? a.cu_seqlens[b] : 0;
  const int n = PROMPT ? min(a.cu_seqlens[b + 1] - lo, a.max_rows) : paged_len(a.cache, b);
  const float* weight = PROMPT ? a.weight + (int64_t)kvh * a.total + lo : a.weight + unit * cap;
  const int32_t* pos = PROMPT ? nullptr : a.pos + unit * cap;
  float* w_out = a.weight_out ? a.weight_out + unit * cap : nullptr;
  int32_t* p_out = a.pos_out + unit * cap;
  const bool copy_w = w_out != nullptr && w_out != weight, copy_p = p_out != pos;
  const int budget = a.budget;
  if (n <= budget) {   // nothing goes
    for (int j = tid; j < n; j += NT) {
      if (copy_w) w_out[j] = weight[j];
      if (copy_p) p_out[j] = PROMPT ? j : pos[j];
    }
    if (!PROMPT && tid == 0) a.n_moves[unit] = 0;
    return;
  }
  // ---- the newest token's position (step form: the largest there is)
  int last = n - 1;
  if (!PROMPT) {
    int m = INT_MIN;
    for (int j = tid; j < n; j += NT) m = max(m, pos[j]);
    m = __reduce_max_sync(0xffffffffu, m);
    if (tid == 0) sh.last = INT_MIN;
    __syncthreads();
    if (lane == 0) atomicMax(&sh.last, m);
    __syncthreads();
    last = sh.last;
  }
  auto key = [&](int j) -> uint32_t {
    const int64_t p = PROMPT ? j : pos[j];
    return (p < a.n_first || p > (int64_t)last - a.n_last) ? KEY_PROTECTED : weight_key(weight[j]);
  };
  // ---- the budget-th largest key
  uint32_t prefix = 0, mask = 0;
  int want = budget;   // how many of the keys that agree with the prefix stay
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < bins; i += NT) sh.hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += NT) {
      const uint32_t u = key(j);
      if ((u & mask) == prefix) atomicAdd(&sh.hist[(u >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // walk the bins from the highest down: thread t owns `per` of them
    const int per = (bins + NT - 1) / NT;
    int mine = 0;
    for (int i = 0; i < per; ++i) {
      const int bin = bins - 1 - (tid * per + i);
      if (bin >= 0) mine += sh.hist[bin];
    }
    int2 total;
    int above = block_exclusive_scan<NT>(make_int2(mine, 0), sh.warp_tot, total).x;
    if (above < want && want <= above + mine) {   // exactly one thread
      for (int i = 0; i < per; ++i) {
        const int bin = bins - 1 - (tid * per + i);
        const int c = sh.hist[bin];
        if (want <= above + c) { sh.bucket = bin; sh.rest = want - above; break; }
        above += c;
      }
    }
    __syncthreads();
    prefix |= (uint32_t)sh.bucket << shift;
    mask |= (uint32_t)(bins - 1) << shift;
    want = sh.rest;
  }
  const uint32_t T = prefix;   // rows with a larger key stay, and the first `want` of those that equal it
  // ---- ranks: warp w owns rows w * seg ..
  const int seg = ((n + NT - 1) / NT) * 32, j0 = warp * seg, j1 = min(j0 + seg, n);
  const uint32_t lt = (1u << lane) - 1u;
  int n_eq = 0;
  for (int j = j0; j < j1; j += 32) {
    const bool eq = j + lane < j1 && key(j + lane) == T;
    n_eq += __popc(__ballot_sync(0xffffffffu, eq));
  }
  int2 total;
  const int eq_base = __shfl_sync(0xffffffffu, block_exclusive_scan<NT>(make_int2(lane == 0 ? n_eq : 0, 0), sh.warp_tot, total).x, 0);
  // x: kept rows (prompt form) or free rows below the budget; y: kept rows behind it
  auto classify = [&](int j, int& eq_seen, bool& x, bool& y, bool& keep) {
    const bool in = j + lane < j1;
    const uint32_t u = in ? key(j + lane) : 0u;
    const uint32_t eqs = __ballot_sync(0xffffffffu, in && u == T);
    keep = in && (u > T || (u == T && eq_seen + __popc(eqs & lt) < want));
    eq_seen += __popc(eqs);
    x = PROMPT ? keep : (in && j + lane < budget && !keep);
    y = !PROMPT && keep && j + lane >= budget;
  };
  int cx = 0, cy = 0, eq_seen = eq_base;
  for (int j = j0; j < j1; j += 32) {
    bool x, y, keep;
    classify(j, eq_seen, x, y, keep);
    cx += __popc(__ballot_sync(0xffffffffu, x));
    cy += __popc(__ballot_sync(0xffffffffu, y));
  }
  int2 base = block_exclusive_scan<NT>(lane == 0 ? make_int2(cx, cy) : make_int2(0, 0), sh.warp_tot, total);
  int rx = __shfl_sync(0xffffffffu, base.x, 0), ry = __shfl_sync(0xffffffffu, base.y, 0);
  const int n_moves = total.y;   // as many free rows as kept rows behind the budget
  int32_t* from = PROMPT ? nullptr : a.moves + (int64_t)unit * 2 * a.list;
  int32_t* to = PROMPT ? nullptr : from + a.list;
  eq_seen = eq_base;
  for (int j = j0; j < j1; j += 32) {
    bool x, y, keep;
    classify(j, eq_seen, x, y, keep);
    const uint32_t bx = __ballot_sync(0xffffffffu, x), by = __ballot_sync(0xffffffffu, y);
    const int me = j + lane;
    if (PROMPT) {
      if (x) {
        const int slot = rx + __popc(bx & lt);
        p_out[slot] = me;
        if (copy_w) w_out[slot] = weight[me];
      }
    } else {
      if (x) to[rx + __popc(bx & lt)] = me;
      if (y) from[ry + __popc(by & lt)] = me;
      if (keep && me < budget) {
        if (copy_w) w_out[me] = weight[me];
        if (copy_p) p_out[me] = pos[me];
      }
    }
    rx += __popc(bx);
    ry += __popc(by);
  }
  if (PROMPT) return;
  __syncthreads();   // the lists are written, and nobody reads a row below the budget any more
  if (tid == 0) a.n_moves[unit] = n_moves;
  for (int i = tid; i < n_moves; i += NT) {
    w_out[to[i]] = weight[from[i]];
    p_out[to[i]] = pos[from[i]];
  }
}

// ---- lists of at most 65536 rows.  A cluster of C CTAs owns a (sequence, kv head); every key is in
// a register (CTA r holds the r-th stretch of the list, a warp a stretch of that, row j0 + 32 i + lane), read once.
// Four digits of 8 bits: each CTA counts a digit's 256 bins in its shared memory (a histogram of its own per digit, cleared
// once; four copies of the first digit's, where every row counts and most fall into a few bins), the counts of the cluster
// are added through distributed shared memory, and the search ends with the first digit whose bin stays whole.  Ranks come
// from one count per warp and one per CTA.  The CTAs then copy the rows they have found themselves (prompt form) or a share
// of the moves (in place), without a second launch where all lists are resident at once.
// In place, a list of at most 4096 rows (one CTA) that is only a few rows too long -- a step's worth -- has them taken out one by
// one instead, by a minimum over the CTA each; a longer list goes through the digits whatever it loses.
// Measured (8 kv heads, bf16, D = 128): 8 prompts of 12000 to 16384 rows to 2048 in 37 us, of which the copies are 20 at 6.7 TB/s
// and the exchanges of the search 7 (fetching the rows that a first digit had settled into L2 meanwhile: 3 us more); 64 lists of
// 8192 rows halved in 38 us; 512 lists of 1025 rows to 1024 in 5.7 us (20 us with 11-bit digits and full scans over the
// CTA, 17 with a search bit by bit).
constexpr int MAX_CLUSTER = 8, MAX_IPT = 16;
constexpr int FEW = 8;           // rows too many that are taken out one by one
// rows of a list a CTA of a cluster is worth (prompt form: 8 x 8 prompts of 2048 rows 34.1 us with 1024 rows each, 24.7 with 512,
// 23.5 with 256; in place, where the moves are fewer: 19.1, 17.3 and 20.4)
constexpr int ROWS_EACH_PROMPT = 256, ROWS_EACH = 512;

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}
// an int of the same place in the shared memory of CTA `rank` of the cluster
__device__ __forceinline__ int peer_int(const int* p, int rank) {
  uint32_t at = (uint32_t)__cvta_generic_to_shared(p);
  int x;
  asm("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}

template <int NT, int IPT>
struct ClusterShared {
  static constexpr int NW = NT / 32;
  int hist[4][256], more[3][256];   // digit d; copies of the first digit's (d = 3)
  int sum[256];                     // the digit's bins over the cluster
  int2 ranks[2][NW];
  int2 cta_total[2];
  int last[NW], cta_last;
  int bin, rest, equal;
  uint32_t low_key[2][NW];
  int low_row[2][NW];
  int src[NT * IPT];                // prompt form: the rows this CTA keeps, in order
};

// sum over the warps in front of this one, CTAs of lower rank included (x, y), and over all of them, of one pair per warp
template <int NW>
__device__ __forceinline__ int2 rank_base(int2 mine, int2* slots, int2* cta_total, int rank, int n_cta, int2& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) slots[warp] = mine;
  __syncthreads();
  const int2 v = lane < NW ? slots[lane] : make_int2(0, 0);
  total = make_int2(__reduce_add_sync(0xffffffffu, v.x), __reduce_add_sync(0xffffffffu, v.y));
  const bool before = lane < warp;
  int2 base = make_int2(__reduce_add_sync(0xffffffffu, before ? v.x : 0), __reduce_add_sync(0xffffffffu, before ? v.y : 0));
  if (n_cta > 1) {
    if (threadIdx.x == 0) *cta_total = total;
    cluster_sync();
    const int2 c = lane < n_cta ? make_int2(peer_int(&cta_total->x, lane), peer_int(&cta_total->y, lane)) : make_int2(0, 0);
    base.x += __reduce_add_sync(0xffffffffu, lane < rank ? c.x : 0);
    base.y += __reduce_add_sync(0xffffffffu, lane < rank ? c.y : 0);
    total = make_int2(__reduce_add_sync(0xffffffffu, c.x), __reduce_add_sync(0xffffffffu, c.y));
  }
  return base;
}

// NT threads a CTA, 1024 of them on an SM
template <int NT, int IPT, bool PROMPT>
__global__ void __launch_bounds__(NT, 1024 / NT) evict_cluster_kernel(EvictArgs a, int n_cta, bool copy_here) {
  constexpr int NW = NT / 32;
  __shared__ ClusterShared<NT, IPT> sh;
  pdl_wait();   // everything below reads or writes global memory
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = n_cta > 1 ? cluster_rank() : 0;
  const int unit = blockIdx.x / n_cta, b = unit / a.Hkv, kvh = unit - b * a.Hkv;
  const int64_t cap = (int64_t)EARN_PAGE_TOKENS * a.cache.pages_per_seq;
  const int lo = PROMPT ? a.cu_seqlens[b] : 0;
  const int n = PROMPT ? min(a.cu_seqlens[b + 1] - lo, a.max_rows) : paged_len(a.cache, b);
  const float* weight = PROMPT ? a.weight + (int64_t)kvh * a.total + lo : a.weight + unit * cap;
  const int32_t* pos = PROMPT ? nullptr : a.pos + unit * cap;
  float* w_out = a.weight_out ? a.weight_out + unit * cap : nullptr;
  int32_t* p_out = a.pos_out + unit * cap;
  const bool copy_w = w_out != nullptr && w_out != weight, copy_p = p_out != pos;
  const int budget = a.budget;
  const int per_cta = ((n + n_cta - 1) / n_cta + 31) / 32 * 32;   // rows of a CTA
  const int c0 = min(rank * per_cta, n), c1 = min(c0 + per_cta, n);
  const int ipt = (c1 - c0 + NT - 1) / NT, j0 = c0 + warp * ipt * 32 + lane;   // this lane's rows: j0 + 32 i < c1, i < ipt
  const int per_row = a.row_bytes / 16, rows_at_once = NT / per_row, part = (tid % per_row) * 16;
  // rows src(i), i0 <= i < i1, of the packed prompt (counted from the sequence's first) -> rows i of the pages
  auto copy_prompt = [&](int i0, int i1, auto src) {
    const char *kp = reinterpret_cast<const char*>(a.k_packed), *vp = reinterpret_cast<const char*>(a.v_packed);
    constexpr int U = 4;   // rows a thread has in flight
    for (int i = i0 + tid / per_row; i < i1; i += U * rows_at_once) {
      uint4 x[U], y[U];
      int64_t dst[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int m = i + k * rows_at_once;
        dst[k] = -1;
        if (m >= i1) continue;
        bool ok;
        const int page = paged_page(a.cache, b, m / EARN_PAGE_TOKENS, ok);
        if (!ok) continue;
        dst[k] = (((int64_t)page * EARN_PAGE_TOKENS + m % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes + part;
        const int64_t at = (((int64_t)lo + src(m)) * a.Hkv + kvh) * a.row_bytes + part;
        x[k] = __ldg(reinterpret_cast<const uint4*>(kp + at));
        y[k] = __ldg(reinterpret_cast<const uint4*>(vp + at));
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (dst[k] < 0) continue;
        *reinterpret_cast<uint4*>(a.cache.k + dst[k]) = x[k];
        *reinterpret_cast<uint4*>(a.cache.v + dst[k]) = y[k];
      }
    }
  };
  if (n <= budget) {   // nothing goes
    for (int j = c0 + tid; j < c1; j += NT) {
      if (copy_w) w_out[j] = weight[j];
      if (copy_p) p_out[j] = PROMPT ? j : pos[j];
    }
    if (PROMPT && copy_here) copy_prompt(c0, c1, [](int m) { return m; });
    if (!PROMPT && !copy_here && rank == 0 && tid == 0) a.n_moves[unit] = 0;
    return;   // (the whole cluster leaves here)
  }
  const bool few = !PROMPT && n_cta == 1 && n - budget <= FEW;   // block-uniform
  if (!few)
    for (int i = tid; i < 7 * 256; i += NT) (&sh.hist[0][0])[i] = 0;
  // ---- keys
  uint32_t u[IPT];
  float w[IPT];
  int p[IPT];
  int last = n - 1;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    const int j = j0 + 32 * i;
    const bool in = i < ipt && j < c1;
    w[i] = in ? weight[j] : 0.f;
    p[i] = PROMPT ? j : in ? pos[j] : INT_MIN;
  }
  if (!PROMPT) {   // the newest token's position
    int m = INT_MIN;
#pragma unroll
    for (int i = 0; i < IPT; ++i) m = max(m, p[i]);
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) sh.last[warp] = m;
  }
  __syncthreads();   // (the histograms are cleared, too)
  if (!PROMPT) {
    last = __reduce_max_sync(0xffffffffu, sh.last[lane % NW]);
    if (n_cta > 1) {
      if (tid == 0) sh.cta_last = last;
      cluster_sync();
      last = __reduce_max_sync(0xffffffffu, lane < n_cta ? peer_int(&sh.cta_last, lane) : INT_MIN);
    }
  }
  const int64_t after = (int64_t)last - a.n_last;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    const bool in = i < ipt && j0 + 32 * i < c1;
    u[i] = !in ? 0u : (p[i] < a.n_first || p[i] > after) ? KEY_PROTECTED : weight_key(w[i]);
  }
  if (few) {
    // ---- the last rows of the order, one by one: the smallest key, and of equal ones the highest row
    int gone[FEW];
#pragma unroll
    for (int m = 0; m < FEW; ++m) {
      gone[m] = INT_MAX;
      if (m >= n - budget) continue;   // block-uniform
      uint32_t low = 0xffffffffu;
      int row = -1;
#pragma unroll
      for (int i = 0; i < IPT; ++i)   // (a lane's rows rise with i; key 0: no row, or one that is out already)
        if (u[i] != 0u && u[i] <= low) { low = u[i]; row = j0 + 32 * i; }
      const uint32_t wlow = __reduce_min_sync(0xffffffffu, low);
      const int wrow = __reduce_max_sync(0xffffffffu, low == wlow ? row : -1);
      if (lane == 0) { sh.low_key[m & 1][warp] = wlow; sh.low_row[m & 1][warp] = wrow; }
      __syncthreads();
      const uint32_t k = lane < NW ? sh.low_key[m & 1][lane] : 0xffffffffu;
      const int r = lane < NW ? sh.low_row[m & 1][lane] : -1;   // (-1: a warp without rows)
      const uint32_t least = __reduce_min_sync(0xffffffffu, r >= 0 ? k : 0xffffffffu);
      gone[m] = __reduce_max_sync(0xffffffffu, k == least ? r : -1);
#pragma unroll
      for (int i = 0; i < IPT; ++i)
        if (j0 + 32 * i == gone[m]) u[i] = 0u;
    }
    // rows below the budget that stay; kept row budget + t moves into the place of its rank's free row
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      const int j = j0 + 32 * i;
      if (u[i] != 0u && j < budget) {
        if (copy_w) w_out[j] = w[i];
        if (copy_p) p_out[j] = p[i];
      }
    }
    int from = -1, to = -1;   // thread t < FEW: row budget + t
    if (tid < FEW && budget + tid < n) {
      from = budget + tid;
      int rank = tid;         // kept rows behind the budget in front of this one
#pragma unroll
      for (int m = 0; m < FEW; ++m) {
        if (gone[m] == budget + tid) from = -1;
        if (gone[m] >= budget && gone[m] < budget + tid) --rank;
      }
#pragma unroll
      for (int m = 0; m < FEW; ++m) {   // the free row with `rank` free rows below it
        int below = 0;
#pragma unroll
        for (int k = 0; k < FEW; ++k) below += gone[k] < gone[m] ? 1 : 0;
        if (gone[m] < budget && below == rank) to = gone[m];
      }
    }
    if (!copy_here && tid == 0) a.n_moves[unit] = 0;   // (the moves are made here all the same)
    // (nobody reads a row below the budget any more: the rows were read ahead of the barriers)
    if (from >= 0) {
      w_out[to] = weight[from];
      p_out[to] = pos[from];
    }
    if (warp == 0) {
      for (int t = 0; t < FEW; ++t) {
        const int f = __shfl_sync(0xffffffffu, from, t), g = __shfl_sync(0xffffffffu, to, t);
        if (f >= 0) move_row(a, b, kvh, f, g, lane, 32);
      }
    }
    return;
  }
  // ---- the budget-th largest key T, digit by digit from the top: `want` of the `equal` keys that agree with T so far stay.
  // (No row's key is 0, so the key 0 of a lane without a row is never counted.)
  uint32_t T = 0;
  int want = budget, equal = 0;
#pragma unroll
  for (int d = 3; d >= 0; --d) {
    if (d < 3 && want == equal) break;   // cluster-uniform: every key that agrees with T stays
    int* hist = d == 3 && (lane & 3) ? sh.more[(lane & 3) - 1] : sh.hist[d];
#pragma unroll
    for (int i = 0; i < IPT; ++i)
      if (u[i] != 0u && (d == 3 || (u[i] >> (8 * d + 8)) == (T >> (8 * d + 8)))) atomicAdd(&hist[(u[i] >> (8 * d)) & 255u], 1);
    __syncthreads();
    int count = 0;
    if (n_cta > 1) {
      if (d == 3 && tid < 256) {
        sh.hist[3][tid] += sh.more[0][tid] + sh.more[1][tid] + sh.more[2][tid];
      }
      cluster_sync();
#pragma unroll
      for (int r = 0; r < MAX_CLUSTER; ++r)
        if (r < n_cta && tid < 256) count += peer_int(&sh.hist[d][tid], r);
    } else if (tid < 256) {
      count = sh.hist[d][tid];
      if (d == 3) count += sh.more[0][tid] + sh.more[1][tid] + sh.more[2][tid];
    }
    if (tid < 256) sh.sum[tid] = count;
    __syncthreads();
    if (warp == 0) {
      // lane l owns bins 255 - 8 l .. 248 - 8 l; the bins of the lanes below it hold larger digits
      int c[8], sum = 0;   // from the largest digit down
#pragma unroll
      for (int k = 0; k < 8; ++k) { c[k] = sh.sum[255 - 8 * lane - k]; sum += c[k]; }
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
      }
      int above = incl - sum;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (above < want && want <= above + c[k]) { sh.bin = 255 - 8 * lane - k; sh.rest = want - above; sh.equal = c[k]; }   // one lane
        above += c[k];
      }
    }
    __syncthreads();
    T |= (uint32_t)sh.bin << (8 * d);
    want = sh.rest;
    equal = sh.equal;
  }
  // ---- rows with a larger key stay, and the first `want` of the `equal` rows that agree with T
  const uint32_t lt = (1u << lane) - 1u;
  uint32_t keep = 0;   // bit i: row j0 + 32 i stays
  int2 total;
  if (want == equal) {   // cluster-uniform
#pragma unroll
    for (int i = 0; i < IPT; ++i) keep |= u[i] >= T && u[i] != 0u ? 1u << i : 0u;
  } else {
    int eq = 0;
#pragma unroll
    for (int i = 0; i < IPT; ++i) eq += __popc(__ballot_sync(0xffffffffu, u[i] == T));
    int seen = rank_base<NW>(make_int2(eq, 0), sh.ranks[0], &sh.cta_total[0], rank, n_cta, total).x;
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      const uint32_t eqs = __ballot_sync(0xffffffffu, u[i] == T);
      if (u[i] > T || (u[i] == T && seen + __popc(eqs & lt) < want)) keep |= 1u << i;
      seen += __popc(eqs);
    }
  }
  // ---- ranks (x: kept rows, or free rows below the budget; y: kept rows behind it)
  auto is_x = [&](int i) { return PROMPT ? (keep >> i & 1u) != 0u : i < ipt && j0 + 32 * i < min(c1, budget) && !(keep >> i & 1u); };
  auto is_y = [&](int i) { return !PROMPT && (keep >> i & 1u) && j0 + 32 * i >= budget; };
  int cx = 0, cy = 0;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    cx += __popc(__ballot_sync(0xffffffffu, is_x(i)));
    if (!PROMPT) cy += __popc(__ballot_sync(0xffffffffu, is_y(i)));
  }
  const int2 base = rank_base<NW>(make_int2(cx, cy), sh.ranks[1], &sh.cta_total[1], rank, n_cta, total);
  int rx = base.x, ry = base.y;
  int32_t* from = PROMPT ? nullptr : a.moves + (int64_t)unit * 2 * a.list;
  int32_t* to = PROMPT ? nullptr : from + a.list;
  // the CTA's first slot: its warp 0's base
  if (PROMPT && tid == 0) sh.bin = base.x;
  if (PROMPT) __syncthreads();
  const int slot0 = PROMPT ? sh.bin : 0;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    const int j = j0 + 32 * i;
    const uint32_t bx = __ballot_sync(0xffffffffu, is_x(i)), by = PROMPT ? 0u : __ballot_sync(0xffffffffu, is_y(i));
    if (PROMPT) {
      if (is_x(i)) {
        const int slot = rx + __popc(bx & lt);
        sh.src[slot - slot0] = j;
        p_out[slot] = j;
        if (copy_w) w_out[slot] = w[i];
      }
    } else {
      if (is_x(i)) to[rx + __popc(bx & lt)] = j;
      if (is_y(i)) from[ry + __popc(by & lt)] = j;
      if ((keep >> i & 1u) && j < budget) {
        if (copy_w) w_out[j] = w[i];
        if (copy_p) p_out[j] = p[i];
      }
    }
    rx += __popc(bx);
    ry += __popc(by);
  }
  if (PROMPT) {
    if (copy_here) __syncthreads();
    int kept = 0;   // by this CTA
#pragma unroll
    for (int k = 0; k < NW; ++k) kept += sh.ranks[1][k].x;
    if (copy_here) copy_prompt(slot0, slot0 + kept, [&](int m) { return sh.src[m - slot0]; });
  } else {
    // the lists are written, and nobody reads a row below the budget any more
    if (n_cta > 1) cluster_sync();
    else __syncthreads();
    const int n_moves = total.y, share = (n_moves + n_cta - 1) / n_cta, i0 = rank * share, i1 = min(i0 + share, n_moves);
    for (int i = i0 + tid; i < i1; i += NT) {
      const int f = from[i], t = to[i];
      w_out[t] = weight[f];
      p_out[t] = pos[f];
    }
    if (!copy_here && rank == 0 && tid == 0) a.n_moves[unit] = n_moves;
    constexpr int U = 4;   // rows a thread has in flight
    for (int i = copy_here ? i0 + tid / per_row : i1; i < i1; i += U * rows_at_once) {
      uint4 x[U], y[U];
      int64_t dst[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int m = i + k * rows_at_once;
        dst[k] = -1;
        if (m >= i1) continue;
        const int f = from[m], t = to[m];
        bool ok_from, ok_to;
        const int pf = paged_page(a.cache, b, f / EARN_PAGE_TOKENS, ok_from), pt = paged_page(a.cache, b, t / EARN_PAGE_TOKENS, ok_to);
        if (!ok_to) continue;
        dst[k] = (((int64_t)pt * EARN_PAGE_TOKENS + t % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes + part;
        const int64_t at = (((int64_t)pf * EARN_PAGE_TOKENS + f % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes + part;
        x[k] = *reinterpret_cast<const uint4*>(a.cache.k + at);
        y[k] = *reinterpret_cast<const uint4*>(a.cache.v + at);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (dst[k] < 0) continue;
        *reinterpret_cast<uint4*>(a.cache.k + dst[k]) = x[k];
        *reinterpret_cast<uint4*>(a.cache.v + dst[k]) = y[k];
      }
    }
  }
  if (n_cta > 1) cluster_sync();   // the other CTAs have read this one's shared memory
}

// The step form's moves, ROWS_PER_CTA of one (sequence, kv head) per CTA; 8, 16 or 32 threads a row
constexpr int ROWS_PER_CTA = 64;

__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int unit = blockIdx.y + gridDim.y * blockIdx.z;
  if (unit >= a.n_seq * a.Hkv) return;
  const int i0 = blockIdx.x * ROWS_PER_CTA, n = min(a.n_moves[unit] - i0, ROWS_PER_CTA);
  if (n <= 0) return;
  const int b = unit / a.Hkv, kvh = unit - b * a.Hkv;
  const int32_t* from = a.moves + (int64_t)unit * 2 * a.list + i0;
  const int32_t* to = from + a.list;
  const int per_row = a.row_bytes / 16, rows_at_once = 256 / per_row;
  for (int i = threadIdx.x / per_row; i < n; i += rows_at_once) move_row(a, b, kvh, from[i], to[i], threadIdx.x % per_row, per_row);
}

// The prompt form's copies: row (cu_seqlens[b] + pos_out[m], kvh) of the packed tensors -> row m of the pages
__global__ void __launch_bounds__(256) evict_gather_kernel(EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int unit = blockIdx.y + gridDim.y * blockIdx.z;
  if (unit >= a.n_seq * a.Hkv) return;
  const int b = unit / a.Hkv, kvh = unit - b * a.Hkv;
  const int lo = a.cu_seqlens[b];
  const int kept = min(min(a.cu_seqlens[b + 1] - lo, a.max_rows), a.budget);
  const int m0 = blockIdx.x * ROWS_PER_CTA, m1 = min(m0 + ROWS_PER_CTA, kept);
  const int64_t cap = (int64_t)EARN_PAGE_TOKENS * a.cache.pages_per_seq;
  const int32_t* src_pos = a.pos_out + unit * cap;
  const char *kp = reinterpret_cast<const char*>(a.k_packed), *vp = reinterpret_cast<const char*>(a.v_packed);
  const int per_row = a.row_bytes / 16, rows_at_once = 256 / per_row;
  const int part = (threadIdx.x % per_row) * 16;
  for (int m = m0 + threadIdx.x / per_row; m < m1; m += rows_at_once) {
    bool ok;
    const int page = paged_page(a.cache, b, m / EARN_PAGE_TOKENS, ok);
    if (!ok) continue;
    const int64_t src = (((int64_t)lo + src_pos[m]) * a.Hkv + kvh) * a.row_bytes + part;
    const int64_t dst = (((int64_t)page * EARN_PAGE_TOKENS + m % EARN_PAGE_TOKENS) * a.Hkv + kvh) * a.row_bytes + part;
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(kp + src)), y = __ldg(reinterpret_cast<const uint4*>(vp + src));
    *reinterpret_cast<uint4*>(a.cache.k + dst) = x;
    *reinterpret_cast<uint4*>(a.cache.v + dst) = y;
  }
}

template <bool PROMPT>
cudaError_t launch_select(const EvictArgs& a, cudaStream_t st) {
  const cudaError_t e = launch_pdl(evict_select_kernel<PROMPT>, dim3((unsigned)a.n_seq * a.Hkv), dim3(SELECT_THREADS), 0, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int NT, int IPT, bool PROMPT>
cudaError_t launch_cluster(const EvictArgs& a, int n_cta, bool copy_here, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.n_seq * a.Hkv * n_cta);
  cfg.blockDim = dim3(NT);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_cta;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = n_cta > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, evict_cluster_kernel<NT, IPT, PROMPT>, a, n_cta, copy_here);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <bool PROMPT>
cudaError_t launch_form(const EvictArgs& a, cudaStream_t st) {
  const int64_t units = (int64_t)a.n_seq * a.Hkv;
  const int excess = a.max_rows > a.budget ? a.max_rows - a.budget : 0;   // rows that go, at most
  bool copied = false;
  cudaError_t e;
  // Threads a CTA.  More of them on a list mean fewer CTAs to a cluster and less waiting for one another (8 prompts of 12000 to
  // 16384 rows 37.2 us with 512, 39.6 with 256); a short list, or one that loses a few rows only, is done sooner by 256
  // (5.6 us against 8.3 for 512 lists of 1025 rows), and more lists than 512-thread CTAs are resident with them.
  constexpr int WIDE = 512, NARROW = 256;
  if (a.max_rows <= MAX_CLUSTER * WIDE * MAX_IPT && units * MAX_CLUSTER <= INT_MAX) {
    // CTAs per list: one if only a few rows go and a CTA's registers hold the list (4096 rows), otherwise as many as leave
    // them ROWS_EACH (_PROMPT) rows while the grid stays within what is resident at once
    int c = 1;
    while (c < MAX_CLUSTER && (a.max_rows > c * (c > 1 ? WIDE : NARROW) * MAX_IPT ||
                               ((PROMPT || excess > FEW) && a.max_rows >= 2 * c * (PROMPT ? ROWS_EACH_PROMPT : ROWS_EACH) &&
                                units * 2 * c <= 1024 / WIDE * sm_count())))
      c *= 2;
    const bool wide = c > 1 || ((PROMPT || excess > FEW) && a.max_rows > 4 * NARROW && units <= 1024 / WIDE * sm_count());
    const int nt = wide ? WIDE : NARROW, per_thread = (a.max_rows + c * nt - 1) / (c * nt);
    // A grid of more than one wave leaves the copies to a kernel of their own: CTAs that come late start copying late (1024
    // lists of 128 to 2048 rows to 512: 97 us in one launch, 92 in two).
    copied = units * c <= 1024 / nt * sm_count() || (!PROMPT && excess <= FEW);
    auto launch = [&](auto nt_tag) {
      constexpr int NT = decltype(nt_tag)::value;
      return per_thread <= 4   ? launch_cluster<NT, 4, PROMPT>(a, c, copied, st)
             : per_thread <= 8 ? launch_cluster<NT, 8, PROMPT>(a, c, copied, st)
                               : launch_cluster<NT, 16, PROMPT>(a, c, copied, st);
    };
    e = wide ? launch(std::integral_constant<int, WIDE>{}) : launch(std::integral_constant<int, NARROW>{});
  } else {
    e = launch_select<PROMPT>(a, st);
  }
  const int kept = a.max_rows < a.budget ? a.max_rows : a.budget;
  const int rows = PROMPT ? kept : excess < a.budget ? excess : a.budget;   // to be copied, or moves, per list at most
  if (e != cudaSuccess || copied || rows == 0) return e;
  const unsigned gy = units < 32768 ? (unsigned)units : 32768u;
  const dim3 grid((rows + ROWS_PER_CTA - 1) / ROWS_PER_CTA, gy, (unsigned)((units + gy - 1) / gy));
  e = PROMPT ? launch_pdl(evict_gather_kernel, grid, dim3(256), 0, st, a) : launch_pdl(evict_move_kernel, grid, dim3(256), 0, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st) {
  return a.k_packed != nullptr ? launch_form<true>(a, st) : launch_form<false>(a, st);
}

}  // namespace earn

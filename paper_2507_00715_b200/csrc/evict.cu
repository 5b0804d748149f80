// Eviction from a cache by accumulated attention weight: which rows of every (sequence, kv head) stay within the budget,
// and their way into (prompt form) or inside (step form) the paged cache.
//
// Selection: one CTA per (sequence, kv head).  Every row gets a 32-bit key that orders as the policy does (a protected
// row the largest key of all, otherwise the weight's bits made monotone), kept in shared memory while the list fits
// there.  The budget-th largest key is found digit by digit (11 + 11 + 10 bits, a histogram in shared memory per
// digit); of the rows that equal it the first ones stay.  Row numbers in order come from ballots: a warp owns a contiguous
// stretch of the list, so a count per warp and one scan over the warps turn into ranks.  Exact, and no result depends on
// the order in which threads arrive.
//   prompt form: the m-th kept position goes to pos_out[m]; a second kernel copies the K / V rows (bit copies, 16-byte
//   vectors) from the packed prompt into the pages.
//   step form: the i-th free row below the budget and the i-th kept row behind it form a move; sources and destinations
//   are disjoint, so the moves run in any order.  A few moves (a step's worth) are made by the selecting CTA itself, more
//   of them by a second kernel over the whole GPU.
#include <climits>

#include "earn_common.cuh"

namespace earn {
namespace {

constexpr int DIGIT_BINS = 2048;
constexpr int STAGE_ROWS = 48 * 1024;   // keys held in shared memory (192 KB); longer lists are read again from L2

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

template <int NT, bool PROMPT, bool STAGED>
__global__ void __launch_bounds__(NT) evict_select_kernel(EvictArgs a, bool move_here) {
  extern __shared__ uint32_t staged[];
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
  auto key_of = [&](int j) -> uint32_t {
    const int64_t p = PROMPT ? j : pos[j];
    return (p < a.n_first || p > (int64_t)last - a.n_last) ? KEY_PROTECTED : weight_key(weight[j]);
  };
  if (STAGED) {
    for (int j = tid; j < n; j += NT) staged[j] = key_of(j);
    __syncthreads();
  }
  auto key = [&](int j) -> uint32_t { return STAGED ? staged[j] : key_of(j); };
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
  if (move_here)
    for (int i = warp; i < n_moves; i += NT / 32) move_row(a, b, kvh, from[i], to[i], lane, 32);
}

// ---- lists of at most NT * IPT rows: every key in a register (row j0 + 32 i + lane of a warp's stretch), read once.
// Four digits of 8 bits: the CTA counts a digit's 256 bins in shared memory (a histogram of its own per digit, so a digit
// costs one barrier) and every warp finds the bin by itself.  Ranks over the warps come from one count per warp and one
// barrier as well.  (Eleven-bit digits and full scans: 20 us for 512 lists of 1025 rows; a search bit by bit: 17 us.)
constexpr int MOVES_HERE = 64;   // moves the selecting CTA makes itself

template <int NT>
struct RegShared {
  int hist[4][256];
  int2 ranks[2][NT / 32];
  int last[NT / 32];
  int from[MOVES_HERE], to[MOVES_HERE];
};

// sum over the warps in front of this one (x, y) and over all of them, of one pair per warp
template <int NW>
__device__ __forceinline__ int2 rank_base(int2 mine, int2* slots, int2& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) slots[warp] = mine;
  __syncthreads();
  const int2 v = lane < NW ? slots[lane] : make_int2(0, 0);
  total = make_int2(__reduce_add_sync(0xffffffffu, v.x), __reduce_add_sync(0xffffffffu, v.y));
  const bool before = lane < warp;
  return make_int2(__reduce_add_sync(0xffffffffu, before ? v.x : 0), __reduce_add_sync(0xffffffffu, before ? v.y : 0));
}

template <int NT, int IPT, bool PROMPT>
__global__ void __launch_bounds__(NT) evict_select_regs_kernel(EvictArgs a, bool move_here) {
  constexpr int NW = NT / 32;
  __shared__ RegShared<NT> sh;
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
  const int ipt = (n + NT - 1) / NT, j0 = warp * ipt * 32 + lane;   // this lane's rows: j0 + 32 i, i < ipt
  if (n <= budget) {   // nothing goes
    for (int j = tid; j < n; j += NT) {
      if (copy_w) w_out[j] = weight[j];
      if (copy_p) p_out[j] = PROMPT ? j : pos[j];
    }
    if (!PROMPT && tid == 0) a.n_moves[unit] = 0;
    return;
  }
  for (int i = tid; i < 4 * 256; i += NT) sh.hist[0][i] = 0;
  // ---- keys
  uint32_t u[IPT];
  int last = n - 1;
  {
    float w[IPT];
    int p[IPT];
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      const int j = j0 + 32 * i;
      const bool in = i < ipt && j < n;
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
    if (!PROMPT) last = __reduce_max_sync(0xffffffffu, sh.last[lane % NW]);
    const int64_t after = (int64_t)last - a.n_last;
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      const bool in = i < ipt && j0 + 32 * i < n;
      u[i] = !in ? 0u : (p[i] < a.n_first || p[i] > after) ? KEY_PROTECTED : weight_key(w[i]);
    }
  }
  // ---- the budget-th largest key T, digit by digit from the top: `want` of the keys that agree with T so far stay.  (No
  // row's key is 0, so the key 0 of a lane without a row is never counted.)
  uint32_t T = 0;
  int want = budget, equal = 0;
#pragma unroll
  for (int d = 3; d >= 0; --d) {
    int* hist = sh.hist[d];
#pragma unroll
    for (int i = 0; i < IPT; ++i)
      if (u[i] != 0u && (d == 3 || (u[i] >> (8 * d + 8)) == (T >> (8 * d + 8)))) atomicAdd(&hist[(u[i] >> (8 * d)) & 255u], 1);
    __syncthreads();
    // lane l owns bins 255 - 8 l .. 248 - 8 l; the bins of the lanes below it hold larger digits
    const int4 h0 = reinterpret_cast<const int4*>(hist)[63 - 2 * lane], h1 = reinterpret_cast<const int4*>(hist)[62 - 2 * lane];
    const int c[8] = {h0.w, h0.z, h0.y, h0.x, h1.w, h1.z, h1.y, h1.x};   // from the largest digit down
    int sum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += c[k];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const int owner = __ffs(__ballot_sync(0xffffffffu, incl >= want)) - 1;
    int above = incl - sum, digit = 0, rest = 0, cnt = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (above < want && want <= above + c[k]) { digit = 255 - 8 * lane - k; rest = want - above; cnt = c[k]; }
      above += c[k];
    }
    T |= (uint32_t)__shfl_sync(0xffffffffu, digit, owner) << (8 * d);
    want = __shfl_sync(0xffffffffu, rest, owner);
    equal = __shfl_sync(0xffffffffu, cnt, owner);
  }
  // ---- rows with a larger key stay, and the first `want` of the `equal` rows with key T
  const uint32_t lt = (1u << lane) - 1u;
  uint32_t keep = 0;   // bit i: row j0 + 32 i stays
  int2 total;
  if (want == equal) {   // block-uniform
#pragma unroll
    for (int i = 0; i < IPT; ++i) keep |= u[i] >= T ? 1u << i : 0u;
  } else {
    int eq = 0;
#pragma unroll
    for (int i = 0; i < IPT; ++i) eq += __popc(__ballot_sync(0xffffffffu, u[i] == T));
    int seen = rank_base<NW>(make_int2(eq, 0), sh.ranks[0], total).x;
#pragma unroll
    for (int i = 0; i < IPT; ++i) {
      const uint32_t eqs = __ballot_sync(0xffffffffu, u[i] == T);
      if (u[i] > T || (u[i] == T && seen + __popc(eqs & lt) < want)) keep |= 1u << i;
      seen += __popc(eqs);
    }
  }
  // ---- ranks (x: kept rows, or free rows below the budget; y: kept rows behind it) and the lists
  auto is_x = [&](int i) { return PROMPT ? (keep >> i & 1u) != 0u : i < ipt && j0 + 32 * i < budget && !(keep >> i & 1u); };
  auto is_y = [&](int i) { return !PROMPT && (keep >> i & 1u) && j0 + 32 * i >= budget; };
  int cx = 0, cy = 0;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    cx += __popc(__ballot_sync(0xffffffffu, is_x(i)));
    if (!PROMPT) cy += __popc(__ballot_sync(0xffffffffu, is_y(i)));
  }
  const int2 base = rank_base<NW>(make_int2(cx, cy), sh.ranks[1], total);
  int rx = base.x, ry = base.y;
  int32_t* from = PROMPT ? nullptr : move_here ? sh.from : a.moves + (int64_t)unit * 2 * a.list;
  int32_t* to = PROMPT ? nullptr : move_here ? sh.to : a.moves + (int64_t)unit * 2 * a.list + a.list;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    if (i >= ipt) break;
    const int j = j0 + 32 * i;
    const uint32_t bx = __ballot_sync(0xffffffffu, is_x(i)), by = PROMPT ? 0u : __ballot_sync(0xffffffffu, is_y(i));
    if (PROMPT) {
      if (is_x(i)) {
        const int slot = rx + __popc(bx & lt);
        p_out[slot] = j;
        if (copy_w) w_out[slot] = weight[j];
      }
    } else {
      if (is_x(i)) to[rx + __popc(bx & lt)] = j;
      if (is_y(i)) from[ry + __popc(by & lt)] = j;
      if ((keep >> i & 1u) && j < budget) {
        if (copy_w) w_out[j] = weight[j];
        if (copy_p) p_out[j] = pos[j];
      }
    }
    rx += __popc(bx);
    ry += __popc(by);
  }
  if (PROMPT) return;
  const int n_moves = total.y;
  __syncthreads();   // the lists are written, and nobody reads a row below the budget any more
  if (tid == NT - 1) a.n_moves[unit] = n_moves;
  for (int i = NT - 1 - tid; i < n_moves; i += NT) {   // (from the last warp down: the first ones move rows meanwhile)
    w_out[to[i]] = weight[from[i]];
    p_out[to[i]] = pos[from[i]];
  }
  if (move_here)
    for (int i = warp; i < n_moves; i += NW) move_row(a, b, kvh, from[i], to[i], lane, 32);
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

template <int NT, bool PROMPT, bool STAGED>
cudaError_t launch_select(const EvictArgs& a, bool move_here, cudaStream_t st) {
  const int smem = STAGED ? (a.max_rows + 3) / 4 * 16 : 0;
  if (STAGED) {
    const cudaError_t e = ensure_dynamic_smem<evict_select_kernel<NT, PROMPT, STAGED>>(STAGE_ROWS * 4);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = launch_pdl(evict_select_kernel<NT, PROMPT, STAGED>, dim3((unsigned)a.n_seq * a.Hkv), dim3(NT), smem, st, a, move_here);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int NT, int IPT, bool PROMPT>
cudaError_t launch_select_regs(const EvictArgs& a, bool move_here, cudaStream_t st) {
  const cudaError_t e = launch_pdl(evict_select_regs_kernel<NT, IPT, PROMPT>, dim3((unsigned)a.n_seq * a.Hkv), dim3(NT), 0, st, a, move_here);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <bool PROMPT>
cudaError_t launch_form(const EvictArgs& a, cudaStream_t st) {
  // the most moves a (sequence, kv head) can need; up to MOVES_HERE are made by the selecting CTA
  const int most = a.max_rows > a.budget ? (a.max_rows - a.budget < a.budget ? a.max_rows - a.budget : a.budget) : 0;
  const bool move_here = !PROMPT && most <= MOVES_HERE;
  cudaError_t e;
  if (a.max_rows > STAGE_ROWS) e = launch_select<1024, PROMPT, false>(a, move_here, st);
  else if (a.max_rows > 1024 * 16) e = launch_select<1024, PROMPT, true>(a, move_here, st);
  else if (a.max_rows > 512 * 16) e = launch_select_regs<1024, 16, PROMPT>(a, move_here, st);
  else if (a.max_rows > 256 * 8) e = launch_select_regs<512, 16, PROMPT>(a, move_here, st);
  else if (a.max_rows > 128 * 4) e = launch_select_regs<256, 8, PROMPT>(a, move_here, st);
  else e = launch_select_regs<128, 4, PROMPT>(a, move_here, st);
  const int rows = PROMPT ? (a.max_rows < a.budget ? a.max_rows : a.budget) : most;
  if (e != cudaSuccess || move_here || rows == 0) return e;
  const unsigned units = (unsigned)a.n_seq * a.Hkv, gy = units < 32768u ? units : 32768u;
  const dim3 grid((rows + ROWS_PER_CTA - 1) / ROWS_PER_CTA, gy, (units + gy - 1) / gy);
  e = PROMPT ? launch_pdl(evict_gather_kernel, grid, dim3(256), 0, st, a) : launch_pdl(evict_move_kernel, grid, dim3(256), 0, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st) {
  return a.k_packed != nullptr ? launch_form<true>(a, st) : launch_form<false>(a, st);
}

}  // namespace earn

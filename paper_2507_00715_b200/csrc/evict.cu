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

// The step form's moves, MOVES_PER_CTA of one (sequence, kv head) per CTA; a warp's lanes are dealt to rows of row_bytes / 16
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
  const int per_row = a.row_bytes / 16, rows_at_once = 256 / per_row;   // 8, 16 or 32 threads a row
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

template <bool PROMPT>
cudaError_t launch_form(const EvictArgs& a, cudaStream_t st) {
  // the most moves a (sequence, kv head) can need; up to 64 are made by the selecting CTA
  const int most = a.max_rows > a.budget ? (a.max_rows - a.budget < a.budget ? a.max_rows - a.budget : a.budget) : 0;
  const bool move_here = !PROMPT && most <= ROWS_PER_CTA;
  cudaError_t e;
  if (a.max_rows > STAGE_ROWS) e = launch_select<1024, PROMPT, false>(a, move_here, st);
  else if (a.max_rows > 2048) e = launch_select<1024, PROMPT, true>(a, move_here, st);
  else e = launch_select<256, PROMPT, true>(a, move_here, st);
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

// How the chunk attention deals its work to the CTAs, computed by every CTA from the device's lengths.
//
// A row tile holds the query rows (token, head) of `tile_tok` consecutive new tokens of one sequence under one head block (the
// query heads of a kv head, or a part of them where a group is larger than a tile).  A work item is `item_tok` tokens (one or
// two row tiles) against every key that its last token sees; its cost is counted in units, one per key tile, with a few in front
// for what an item takes besides.  The units of all
// items, in the order (sequence, head block, item, key tile), form one line, which is cut into equal shares, one per CTA: long
// lists are split over CTAs, short ones share one, whatever the mix of single tokens and long chunks.  A cut that falls close
// to an item's edge is moved there, so that only cuts that pay make partial results.
//
// Several items of the same keys (a long chunk) should be worked on at the same time, or every one of them brings the keys from
// HBM again.  So where there are at least four of them on average, and two items per CTA, the line runs through the items by
// columns: item i of the order above stands in column i % CTAs, and a column's items follow one another.  A CTA's share is then
// about one column, and neighbouring CTAs are at neighbouring items.  (8 sequences of 1024 new tokens over 16000-31000 rows, 32/8
// heads: 3524 us by the line, 3324 by columns; 8 prompts of 4096: 1302 and 1186.)
//
// All of it is whole-number arithmetic on the lengths, in 32 bits (a call with 2^31 units or more is refused): every CTA finds
// its own share and, for an item in parts, who else holds one, without a planning kernel.
#pragma once
#include <stdint.h>

namespace earn {

struct ChunkSeq {
  int tok0, n, base;   // first new token, new tokens, rows in front of them (negative: the first new tokens have no row)
  int items;           // under one head block
};
struct ChunkSched {
  const int32_t* cu_new;    // [n_seq + 1] offsets of the sequences' new tokens
  const int32_t* seq_len;   // [n_seq] rows with the new ones
  int n_seq, n_tokens, max_len;
  int heads;                // head blocks: Hkv * ceil(g / heads of a block)
  int item_tok, key_shift;  // tokens of an item; keys of a key tile, as a power of two
  int item_cost, free_tok;  // units at the beginning of an item that stand for no key tile; items of up to free_tok tokens have none
  int grid, min_share;      // CTAs launched; units a CTA takes at least
  const ChunkSeq* table;    // the sequences, where a CTA has them in shared memory (up to kChunkTable), or null
  const int* first;         // with columns: every sequence's first item in the order above, and their number
};
constexpr int kChunkTable = 960, kChunkFirst = 64;   // columns: of up to kChunkFirst sequences

// Offsets that run past the batch or backwards are cut off, so that no row outside q and o is touched: lo to where it belongs.
__host__ __device__ inline int chunk_new(const ChunkSched& s, int& lo, int hi) {   // returns the new tokens
  lo = lo < 0 ? 0 : lo > s.n_tokens ? s.n_tokens : lo;
  hi = hi < lo ? lo : hi > s.n_tokens ? s.n_tokens : hi;
  return hi - lo;
}
__host__ __device__ inline ChunkSeq chunk_seq(const ChunkSched& s, int b) {
  if (s.table != nullptr) return s.table[b];
  ChunkSeq q;
  int lo = s.cu_new[b], len = s.seq_len[b];
  q.n = chunk_new(s, lo, s.cu_new[b + 1]);
  len = len < 0 ? 0 : len > s.max_len ? s.max_len : len;
  q.tok0 = lo; q.base = len - q.n;
  q.items = (q.n + s.item_tok - 1) / s.item_tok;
  return q;
}
// keys that the tokens of item m see between them
__host__ __device__ inline int chunk_keys(const ChunkSched& s, const ChunkSeq& q, int m) {
  const int64_t end = (int64_t)(m + 1) * s.item_tok;
  const int seen = q.base + (int)(end < q.n ? end : q.n);
  return seen > 0 ? seen : 0;
}
__host__ __device__ inline int chunk_cost(const ChunkSched& s, const ChunkSeq& q, int m) { return q.n - m * s.item_tok <= s.free_tok ? 0 : s.item_cost; }
// units of item m: at least one with a key tile, so that rows that see nothing are written too
__host__ __device__ inline int chunk_units(const ChunkSched& s, const ChunkSeq& q, int m) {
  const int u = (chunk_keys(s, q, m) + (1 << s.key_shift) - 1) >> s.key_shift;
  return (u > 0 ? u : 1) + chunk_cost(s, q, m);
}
// sum over i < n of floor((a i + b) / 2^shift), by the Euclidean recursion; a n + b and the sum below 2^32
__host__ __device__ inline uint32_t floor_sum(uint32_t n, int shift, uint32_t a, uint32_t b) {
  const uint32_t mask = (1u << shift) - 1;
  uint32_t sum = (uint32_t)((uint64_t)n * (n - 1) / 2) * (a >> shift) + n * (b >> shift);
  a &= mask;
  b &= mask;
  uint32_t y = a * n + b, m = 1u << shift;
  if (y < m) return sum;
  n = y >> shift;
  b = y & mask;
  while (true) {   // the rows of the triangle instead of its columns: m and a change places
    const uint32_t t = m;
    m = a;
    a = t;
    uint32_t k = a / m;
    sum += (uint32_t)((uint64_t)n * (n - 1) / 2) * k;
    a -= k * m;
    if (b >= m) {
      k = b / m;
      sum += n * k;
      b -= k * m;
    }
    y = a * n + b;
    if (y < m) return sum;
    n = y / m;
    b = y - n * m;
  }
}
// units of the first `count` items of a sequence under one head block
__host__ __device__ inline uint32_t chunk_units_before(const ChunkSched& s, const ChunkSeq& q, int count) {
  const int items = q.items;
  if (count == 1 || items == 1) return count > 0 ? chunk_units(s, q, 0) : 0;
  int whole = count < items ? count : items - 1;   // items whose end is a multiple of item_tok
  if (whole < 0) whole = 0;
  uint32_t sum = whole * s.item_cost;   // (free_tok < item_tok)
  int skip = 0;
  if (q.base < 0) {   // leading items that see less than one key
    skip = (int)((1 - (int64_t)q.base + s.item_tok - 1) / s.item_tok) - 1;
    skip = skip < whole ? skip : whole;
    sum += skip;
  }
  if (whole > skip)
    sum += floor_sum(whole - skip, s.key_shift, s.item_tok, (uint32_t)(q.base + (int64_t)(skip + 1) * s.item_tok + (1 << s.key_shift) - 1));
  if (count >= items && items > 0) sum += chunk_units(s, q, items - 1);
  return sum;
}

struct ChunkWalk {
  uint32_t pos, end;    // units of the line: next one, and the end of this CTA's share
  uint32_t total, tol;  // units in all; a cut closer than this to an item's edge is moved there
  int shares;           // shares the line is cut into: share c begins at c * quot + c * rem / shares
  uint32_t quot, rem;
  int b, h, m, off;     // where pos is: unit `off` of item m under head block h of sequence b
  int cols, col, i;     // columns of the line (1: the items' own order), the one that pos is in, and that item's number in the order
};
__host__ __device__ inline void chunk_cuts(const ChunkSched& s, ChunkWalk& w) {
  const uint32_t shares = (w.total + s.min_share - 1) / s.min_share;
  w.shares = (int)(shares < (uint32_t)s.grid ? (shares > 0 ? shares : 1) : (uint32_t)s.grid);
  w.quot = w.total / w.shares;
  w.rem = w.total - w.quot * w.shares;
  // (a part more costs its writing and the join, about three key tiles' worth of time)
  const uint32_t few = w.quot / 6 < 3 ? w.quot / 6 : 3;
  w.tol = w.quot / 16 > few ? w.quot / 16 : few;
}
__host__ __device__ inline uint32_t chunk_cut(const ChunkWalk& w, int c) { return c * w.quot + c * w.rem / w.shares; }

// w to the item that stands at w.i in the order (sequence, head block, item); w.b = n_seq behind the last one
__host__ __device__ inline void chunk_place(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q) {
  if (w.i >= s.first[s.n_seq]) { w.b = s.n_seq; return; }
  int b = 0;
  for (int step = kChunkFirst / 2; step > 0; step >>= 1)
    if (b + step < s.n_seq && s.first[b + step] <= w.i) b += step;   // the last one that starts there or before: it is not empty
  w.b = b;
  q = chunk_seq(s, b);
  const int at = w.i - s.first[b];
  w.h = at / q.items;
  w.m = at - w.h * q.items;
}
// the item that follows on the line
__host__ __device__ inline void chunk_next(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q) {
  w.off = 0;
  if (w.cols > 1) {
    w.i += w.cols;
    if (w.i >= s.first[s.n_seq] && w.col + 1 < w.cols) w.i = ++w.col;
    chunk_place(s, w, q);
    return;
  }
  if (++w.m < q.items) return;
  w.m = 0;
  if (++w.h < s.heads) return;
  w.h = 0;
  do {
    if (++w.b >= s.n_seq) return;
    q = chunk_seq(s, w.b);
  } while (q.n == 0);
}
// Moves unit x of the line, which lies at unit w.off of the item where w is, to the item's edge where it is close to one.
// Returns the cut; w moves with it.
__host__ __device__ inline uint32_t chunk_settle(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q, uint32_t x) {
  const uint32_t off = w.off, cost = chunk_cost(s, q, w.m), left = chunk_units(s, q, w.m) - off;
  if (off <= w.tol + cost) {
    w.off = 0;
    return x - off;
  }
  if (left > w.tol) return x;
  chunk_next(s, w, q);
  return x + left;
}
// Own order (w.cols = 1): w to unit `r` of sequence b's items under its head block h.
__host__ __device__ inline void chunk_find(const ChunkSched& s, ChunkWalk& w, const ChunkSeq& q, uint32_t r) {
  int lo = 0, hi = q.items;   // the last item that starts at or before r lies in lo .. hi - 1
#ifdef __CUDA_ARCH__
  while (hi - lo > 1) {       // (the whole warp: 32 places at once)
    const int step = (hi - lo + 31) / 32, mine = lo + (int)(threadIdx.x & 31) * step;
    const uint32_t starts = __ballot_sync(0xffffffffu, mine < hi && chunk_units_before(s, q, mine) <= r);
    lo += (31 - __clz(starts)) * step;
    hi = hi < lo + step ? hi : lo + step;
  }
#else
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (chunk_units_before(s, q, mid) <= r) lo = mid; else hi = mid;
  }
#endif
  w.m = lo;
  w.off = lo > 0 ? (int)(r - chunk_units_before(s, q, lo)) : (int)r;
}

// An item in parts: CTAs first .. first + parts - 1 hold one each (parts = 1: the item is whole).
struct ChunkParts {
  int first, parts;
};
// the first cut at or behind unit y
__host__ __device__ inline int chunk_cut_from(const ChunkWalk& w, uint32_t y) {
  int c = (int)((float)y * ((float)w.shares / (float)w.total));
  c = c < w.shares ? c : w.shares;
  while (c > 0 && chunk_cut(w, c - 1) >= y) --c;
  while (chunk_cut(w, c) < y) ++c;
  return c;
}
__host__ __device__ inline ChunkParts chunk_parts(const ChunkWalk& w, uint32_t start, int units, int cost) {
  ChunkParts p{0, 1};
  if ((uint32_t)units <= 2 * w.tol + cost + 1) return p;
  const int lo = chunk_cut_from(w, start + cost + w.tol + 1), hi = chunk_cut_from(w, start + units - w.tol) - 1;   // cuts further than tol inside
  p.parts = hi >= lo ? hi - lo + 2 : 1;
  p.first = lo - 1;
  return p;
}

// columns of the line, see above; `threads`: a column's units are summed up by a thread or several
__host__ __device__ inline int chunk_columns(uint32_t items, uint32_t lists, int n_seq, int shares, int threads) {
  return shares <= threads && n_seq <= kChunkFirst && items >= 2u * shares && items / 4 >= lists ? shares : 1;
}

#ifdef __CUDACC__
struct ChunkCounts {
  uint32_t units;
  int items, lists;   // of sequences
};
// Which of the two bf16 kernels a call belongs to: the one for many rows if a sequence has more than `few` new tokens and the
// other one would have more than `units` products of 16 rows and a key tile under a head block (its items times the tiles of
// their list).
struct ChunkSplit {
  int few, units;
  int item_tok;   // tokens of an item of the other kernel
  int known;      // the lengths need not be looked at: it is the other kernel's
};
// The same answer in every thread of every block, and in both kernels.
__device__ inline bool chunk_many(const ChunkSched& s, const ChunkSplit& f) {
  __shared__ uint32_t sum;
  if (f.known) return false;
  if (threadIdx.x == 0) sum = 0;
  bool longer = false;
  uint32_t mine = 0;
  for (int b = threadIdx.x; b < s.n_seq; b += blockDim.x) {
    int lo = s.cu_new[b];
    const int n = chunk_new(s, lo, s.cu_new[b + 1]), len = s.seq_len[b];
    longer |= n > f.few;
    const int tiles = ((len < s.max_len ? len : s.max_len) + 127) >> 7;
    const uint64_t units = (uint64_t)((n + f.item_tok - 1) / f.item_tok) * (tiles > 0 ? tiles : 1);
    mine += (uint32_t)(units < 65535 ? units : 65535);   // (at most 65535 sequences: 32 bits hold the sum)
  }
  if (!__syncthreads_or(longer)) return false;
  mine = __reduce_add_sync(0xffffffffu, mine);
  if ((threadIdx.x & 31) == 0) atomicAdd(&sum, mine);
  __syncthreads();
  return sum > (uint32_t)f.units;
}
// Sums (units, items, lists) over the block; returns the units of the threads in front of this one.  2^31 units or more, which
// only offsets that run backwards can make (tokens that belong to several sequences): no units.
__device__ inline uint32_t chunk_scan(ChunkCounts& c, int4* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  uint32_t incl = c.units;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += v;
  }
  const uint32_t inside = incl - c.units;
  const int items = __reduce_add_sync(0xffffffffu, c.items), lists = __reduce_add_sync(0xffffffffu, c.lists);
  const uint32_t high = __reduce_add_sync(0xffffffffu, c.units >> 16);   // (65536 units each: what the sum would be without its 32 bits)
  __syncthreads();
  if (lane == 31) scratch[warp] = make_int4((int)incl, items, lists, (int)high);
  __syncthreads();
  const int4 n = lane < warps ? scratch[lane] : make_int4(0, 0, 0, 0);
  uint32_t sum = (uint32_t)n.x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += v;
  }
  c.units = __reduce_add_sync(0xffffffffu, (uint32_t)n.w) < 32768u ? __shfl_sync(0xffffffffu, sum, 31) : 0u;
  c.items = __reduce_add_sync(0xffffffffu, n.y);
  c.lists = __reduce_add_sync(0xffffffffu, n.z);
  return __shfl_sync(0xffffffffu, sum - (uint32_t)n.x, warp) + inside;
}

// This CTA's share of the line; every thread of the CTA calls it (`scratch`: 16-byte aligned shared memory for 48 16-byte words;
// `table`: for kChunkTable sequences, or null).  From then on s reads the sequences from the table, where they fit.
__device__ inline ChunkWalk chunk_share(ChunkSched& s, int4* scratch, ChunkSeq* table) {
  const int t = threadIdx.x, threads = blockDim.x, c = blockIdx.x;
  const bool in_table = table != nullptr && s.n_seq <= kChunkTable;
  const int per = s.n_seq <= threads ? 1 : (s.n_seq + threads - 1) / threads, b0 = min(t * per, s.n_seq), b1 = min(b0 + per, s.n_seq);
  ChunkCounts n{};
  uint64_t units = 0;
  for (int b = b0; b < b1; ++b) {
    const ChunkSeq q = chunk_seq(s, b);
    if (in_table) table[b] = q;
    if (q.n == 0) continue;
    n.items += q.items;
    ++n.lists;
    units += s.heads * chunk_units_before(s, q, q.items);
  }
  n.units = (uint32_t)(units < 0x80000000u ? units : 0x80000000u);
  int own_items = n.items;
  uint32_t mine = n.units, before = chunk_scan(n, scratch);
  if (in_table) s.table = table;   // (written in front of the scan's barriers)
  ChunkWalk w{};
  w.total = n.units;
  if (n.units == 0) return w;
  chunk_cuts(s, w);
  w.cols = in_table ? chunk_columns((uint32_t)n.items * s.heads, (uint32_t)n.lists * s.heads, s.n_seq, w.shares, threads) : 1;
  int each = 1;   // threads of a column, a power of two
  if (w.cols > 1) {
    int* first = reinterpret_cast<int*>(table + kChunkFirst);
    if (t < kChunkFirst) {   // (a sequence a thread)
      int incl = own_items;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, d);
        if ((t & 31) >= d) incl += v;
      }
      if (t >= 32) incl += scratch[0].y;   // (the first warp's items)
      if (t < s.n_seq) first[t + 1] = incl * s.heads;
      if (t == 0) first[0] = 0;
    }
    s.first = first;
    __syncthreads();
    const int items = n.items * s.heads;
    while (each < 32 && 2 * each * w.cols <= threads) each *= 2;
    ChunkCounts col{};
    if (t < w.cols * each) {
      ChunkWalk v = w;
      ChunkSeq q;
      for (v.i = t / each + t % each * w.cols; v.i < items; v.i += each * w.cols) {
        chunk_place(s, v, q);
        col.units += chunk_units(s, q, v.m);
      }
    }
    for (int d = 1; d < each; d <<= 1) col.units += __shfl_xor_sync(0xffffffffu, col.units, d);
    if (t % each != 0) col.units = 0;
    mine = col.units;
    before = chunk_scan(col, scratch);
  }
  // who knows where the cuts lie says so, and a warp each finds the place
  const uint32_t x0 = chunk_cut(w, c), x1 = chunk_cut(w, c + 1);
  uint32_t* place = reinterpret_cast<uint32_t*>(scratch + 32);   // two of: thread's number, units in front of it
  if (c < w.shares && mine > 0) {
    if (x0 >= before && x0 < before + mine) { place[0] = t; place[1] = before; }
    if (x1 >= before && x1 < before + mine) { place[2] = t; place[3] = before; }
  }
  __syncthreads();
  uint32_t* found = place + 4;
  if (t < 64) {
    const int side = t >> 5;
    const uint32_t x = side ? x1 : x0;
    ChunkWalk v = w;
    uint32_t cut = w.total;
    if (c < w.shares && x < w.total) {
      const int owner = (int)place[2 * side];
      uint32_t at = place[2 * side + 1];
      ChunkSeq q;
      if (w.cols > 1) {
        v.col = owner / each;
        for (int i = v.col;; i += 32 * w.cols) {   // (32 of the column's items at once)
          v.i = i + (t & 31) * w.cols;
          chunk_place(s, v, q);
          const uint32_t u = v.b < s.n_seq ? chunk_units(s, q, v.m) : 0;
          uint32_t incl = u;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
            if ((t & 31) >= d) incl += y;
          }
          const uint32_t behind = __ballot_sync(0xffffffffu, at + incl > x);
          if (behind == 0) {
            at += __shfl_sync(0xffffffffu, incl, 31);
            continue;
          }
          const int lane = __ffs(behind) - 1;
          at += __shfl_sync(0xffffffffu, incl - u, lane);
          v.i = i + lane * w.cols;
          break;
        }
        chunk_place(s, v, q);
        v.off = (int)(x - at);
      } else {
        for (v.b = owner * per;; ++v.b) {
          q = chunk_seq(s, v.b);
          if (q.n == 0) continue;
          const uint32_t per_head = chunk_units_before(s, q, q.items);
          if (x < at + s.heads * per_head) {
            v.h = (int)((x - at) / per_head);
            chunk_find(s, v, q, x - at - v.h * per_head);
            break;
          }
          at += s.heads * per_head;
        }
      }
      cut = chunk_settle(s, v, q, x);
    }
    if ((t & 31) == 0) {
      found[side] = cut;
      if (side == 0) { found[2] = v.b; found[3] = v.h; found[4] = v.m; found[5] = v.off; found[6] = v.col; found[7] = v.i; }
    }
  }
  __syncthreads();
  w.pos = found[0]; w.end = found[1];
  w.b = (int)found[2]; w.h = (int)found[3]; w.m = (int)found[4]; w.off = (int)found[5]; w.col = (int)found[6]; w.i = (int)found[7];
  __syncthreads();
  return w;
}
#endif

}  // namespace earn

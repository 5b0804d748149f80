// How the chunk attention deals its work to the CTAs, computed by every CTA from the device's lengths.
//
// A row tile holds the query rows (token, head) of `tile_tok` consecutive new tokens of one sequence under one head block (the
// query heads of a kv head, or a part of them where a group is larger than a tile).  A work item is `item_tok` tokens (one or
// two row tiles) against every key that its last token sees; its cost is counted in units, one per key tile.  The units of all
// items, in the order (sequence, head block, item, key tile), form one line, which is cut into equal shares, one per CTA: long
// lists are split over CTAs, short ones share one, whatever the mix of single tokens and long chunks.  A cut that falls close
// to an item's edge is moved there, so that only cuts that pay make partial results.
//
// Several items of the same keys (a long chunk) should be worked on at the same time, or every one of them brings the keys from
// HBM again.  So where there are at least four of them on average, and two items per CTA, the line runs through the items by
// columns: item i of the order above stands in column i % CTAs, and a column's items follow one another.  A CTA's share is then
// about one column, and neighbouring CTAs are at neighbouring items.  (8 sequences of 1024 new tokens over 16000-31000 rows:
// DRAM traffic 13.4 -> 1.9 GB a layer.)  All of it is whole-number arithmetic on
// the lengths: every CTA finds its own share and, for an item in parts, who else holds one, without a planning kernel.
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
  int item_tok, key_tile;
  int grid, min_share;      // CTAs launched; units a CTA takes at least
  const ChunkSeq* table;    // the sequences, where a CTA has them in shared memory (up to kChunkTable), or null
};
constexpr int kChunkTable = 1024;

// Offsets that run past the batch or backwards are cut off, so that no row outside q and o is touched.
__host__ __device__ inline ChunkSeq chunk_seq(const ChunkSched& s, int b) {
  if (s.table != nullptr) return s.table[b];
  ChunkSeq q;
  int lo = s.cu_new[b], hi = s.cu_new[b + 1], len = s.seq_len[b];
  lo = lo < 0 ? 0 : lo > s.n_tokens ? s.n_tokens : lo;
  hi = hi < lo ? lo : hi > s.n_tokens ? s.n_tokens : hi;
  len = len < 0 ? 0 : len > s.max_len ? s.max_len : len;
  q.tok0 = lo; q.n = hi - lo; q.base = len - q.n;
  q.items = (q.n + s.item_tok - 1) / s.item_tok;
  return q;
}
// keys that the tokens of item m see between them
__host__ __device__ inline int chunk_keys(const ChunkSched& s, const ChunkSeq& q, int m) {
  const int64_t end = (int64_t)(m + 1) * s.item_tok;
  const int seen = q.base + (int)(end < q.n ? end : q.n);
  return seen > 0 ? seen : 0;
}
// units of item m: at least one, so that rows that see nothing are written too
__host__ __device__ inline int chunk_units(const ChunkSched& s, const ChunkSeq& q, int m) {
  const int u = (chunk_keys(s, q, m) + s.key_tile - 1) / s.key_tile;
  return u > 0 ? u : 1;
}
// sum over i < n of floor((a i + b) / m), by the Euclidean recursion; a n + b below 2^32
__host__ __device__ inline int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  int64_t sum = 0;
  while (true) {
    if (a >= m) { const uint32_t k = a / m; sum += (int64_t)n * (n - 1) / 2 * k; a -= k * m; }
    if (b >= m) { const uint32_t k = b / m; sum += (int64_t)n * k; b -= k * m; }
    const uint32_t y = a * n + b;
    if (y < m) return sum;
    n = y / m;
    b = y - n * m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
}
// units of the first `count` items of a sequence under one head block
__host__ __device__ inline int64_t chunk_units_before(const ChunkSched& s, const ChunkSeq& q, int count) {
  const int items = q.items;
  if (count == 1 || items == 1) return count > 0 ? chunk_units(s, q, 0) : 0;
  int whole = count < items ? count : items - 1;   // items whose end is a multiple of item_tok
  if (whole < 0) whole = 0;
  int64_t sum = 0;
  int skip = 0;
  if (q.base < 0) {   // leading items that see less than one key
    skip = (int)((1 - (int64_t)q.base + s.item_tok - 1) / s.item_tok) - 1;
    skip = skip < whole ? skip : whole;
    sum += skip;
  }
  if (whole > skip)
    sum += floor_sum(whole - skip, s.key_tile, s.item_tok, (uint32_t)(q.base + (int64_t)(skip + 1) * s.item_tok + s.key_tile - 1));
  if (count >= items && items > 0) sum += chunk_units(s, q, items - 1);
  return sum;
}

struct ChunkWalk {
  int64_t pos, end;    // units of the line: next one, and the end of this CTA's share
  int64_t total, tol;  // units in all; a cut closer than this to an item's edge is moved there
  int shares;          // shares the line is cut into
  int b, h, m, off;    // where pos is: unit `off` of item m under head block h of sequence b
  int longest;         // most new tokens of a sequence
  int cols, col;       // columns of the line (1: the items' own order), and the one that pos is in
};

__host__ __device__ inline int64_t chunk_cut(const ChunkWalk& w, int c) { return (int64_t)c * w.total / w.shares; }

// `count` items further in the order (sequence, head block, item); w.b = n_seq behind the last one
__host__ __device__ inline void chunk_skip(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q, int count) {
  if (w.m + count < q.items) { w.m += count; return; }
  int64_t at = (int64_t)w.h * q.items + w.m + count, all;
  while (at >= (all = (int64_t)s.heads * q.items)) {
    at -= all;
    do {
      if (++w.b >= s.n_seq) return;
      q = chunk_seq(s, w.b);
    } while (q.n == 0);
  }
  w.h = (int)(at / q.items);
  w.m = (int)(at - (int64_t)w.h * q.items);
}
// the first item of a column (there is one: no more columns than items)
__host__ __device__ inline void chunk_column(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q, int col) {
  w.col = col;
  w.h = w.m = w.off = w.b = 0;
  for (q = chunk_seq(s, 0); q.n == 0; q = chunk_seq(s, w.b)) ++w.b;
  chunk_skip(s, w, q, col);
}
// the item that follows on the line
__host__ __device__ inline void chunk_next(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q) {
  w.off = 0;
  chunk_skip(s, w, q, w.cols);
  if (w.b >= s.n_seq && w.col + 1 < w.cols) chunk_column(s, w, q, w.col + 1);
}
// Moves unit x of the line, which lies at unit w.off of the item where w is, to the item's edge where it is close to one.
// Returns the cut; w moves with it.
__host__ __device__ inline int64_t chunk_settle(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q, int64_t x) {
  const int off = w.off, left = chunk_units(s, q, w.m) - off;
  if (off <= w.tol) {
    w.off = 0;
    return x - off;
  }
  if (left > w.tol) return x;
  chunk_next(s, w, q);
  return x + left;
}
// Own order (w.cols = 1): w to unit `r` of sequence b's items under its head block h.
__host__ __device__ inline void chunk_find(const ChunkSched& s, ChunkWalk& w, const ChunkSeq& q, int64_t r) {
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
  w.off = (int)(r - chunk_units_before(s, q, lo));
}

// An item in parts: CTAs first .. first + parts - 1 hold one each (parts = 1: the item is whole).
struct ChunkParts {
  int first, parts;
};
__host__ __device__ inline ChunkParts chunk_parts(const ChunkWalk& w, int64_t start, int units) {
  const int64_t g = w.shares, u = w.total;
  const int64_t lo = ((start + w.tol + 1) * g + u - 1) / u;            // first cut more than tol behind the start
  const int64_t hi = ((start + units - w.tol) * g + u - 1) / u - 1;    // last cut more than tol in front of the end
  ChunkParts p;
  p.parts = hi >= lo ? (int)(hi - lo) + 2 : 1;
  p.first = (int)lo - 1;
  return p;
}

// columns of the line, see above; `threads`: a column's units are summed up by a thread
__host__ __device__ inline int chunk_columns(int64_t items, int64_t lists, int n_seq, int shares, int threads) {
  return shares <= threads && n_seq <= 64 && items >= 2 * (int64_t)shares && items >= 4 * lists ? shares : 1;
}

#ifdef __CUDACC__
struct ChunkCounts {
  int64_t units;
  int items, lists, longest;   // (items and lists: of sequences)
};
// Sums (units, items, lists) and maximum (longest) over the block; returns the units of the threads in front of this one.
__device__ inline int64_t chunk_scan(ChunkCounts& c, int64_t* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  int64_t incl = c.units;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += v;
  }
  const int64_t inside = incl - c.units;
  c.items = __reduce_add_sync(0xffffffffu, c.items);
  c.lists = __reduce_add_sync(0xffffffffu, c.lists);
  c.longest = __reduce_max_sync(0xffffffffu, c.longest);
  __syncthreads();
  if (lane == 31) {
    scratch[warp] = incl;
    reinterpret_cast<int4*>(scratch + 32)[warp] = make_int4(c.items, c.lists, c.longest, 0);
  }
  __syncthreads();
  const int64_t mine = lane < warps ? scratch[lane] : 0;
  const int4 n = lane < warps ? reinterpret_cast<int4*>(scratch + 32)[lane] : make_int4(0, 0, 0, 0);
  int64_t sum = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += v;
  }
  c.units = __shfl_sync(0xffffffffu, sum, 31);
  c.items = __reduce_add_sync(0xffffffffu, n.x);
  c.lists = __reduce_add_sync(0xffffffffu, n.y);
  c.longest = __reduce_max_sync(0xffffffffu, n.z);
  return __shfl_sync(0xffffffffu, sum - mine, warp) + inside;
}

// This CTA's share of the line; every thread of the CTA calls it (`scratch`: 16-byte aligned shared memory for 96 64-bit words;
// `table`: for kChunkTable sequences, or null).  From then on s reads the sequences from the table, where they fit.
__device__ inline ChunkWalk chunk_share(ChunkSched& s, int64_t* scratch, ChunkSeq* table) {
  const int t = threadIdx.x, threads = blockDim.x, c = blockIdx.x;
  const bool in_table = table != nullptr && s.n_seq <= kChunkTable;
  const int per = (s.n_seq + threads - 1) / threads, b0 = min(t * per, s.n_seq), b1 = min(b0 + per, s.n_seq);
  ChunkCounts n{};
  for (int b = b0; b < b1; ++b) {
    const ChunkSeq q = chunk_seq(s, b);
    if (in_table) table[b] = q;
    if (q.n == 0) continue;
    n.longest = max(n.longest, q.n);
    n.items += q.items;
    ++n.lists;
    n.units += s.heads * chunk_units_before(s, q, q.items);
  }
  int64_t mine = n.units, before = chunk_scan(n, scratch);
  if (in_table) s.table = table;   // (written in front of the scan's barriers)
  ChunkWalk w{};
  w.total = n.units;
  w.longest = n.longest;
  const int64_t shares = (w.total + s.min_share - 1) / s.min_share;
  w.shares = (int)(shares < s.grid ? (shares > 0 ? shares : 1) : s.grid);
  w.tol = w.total / (w.shares * 16);
  w.cols = chunk_columns((int64_t)n.items * s.heads, (int64_t)n.lists * s.heads, s.n_seq, w.shares, threads);
  if (w.cols > 1) {
    ChunkCounts col{};
    if (t < w.cols) {
      ChunkWalk v = w;
      ChunkSeq q;
      for (chunk_column(s, v, q, t); v.b < s.n_seq; chunk_skip(s, v, q, w.cols)) col.units += chunk_units(s, q, v.m);
    }
    mine = col.units;
    before = chunk_scan(col, scratch);
  }
  // who knows where the cuts lie says so, and a warp each finds the place
  const int64_t x0 = chunk_cut(w, c), x1 = chunk_cut(w, c + 1);
  int64_t* place = scratch + 80;   // [2]: first thread's number and units in front of it
  if (c < w.shares && mine > 0) {
    if (x0 >= before && x0 < before + mine) { place[0] = t; place[1] = before; }
    if (x1 >= before && x1 < before + mine) { place[2] = t; place[3] = before; }
  }
  __syncthreads();
  int64_t* found = scratch + 84;
  if (t < 64) {
    const int side = t >> 5;
    const int64_t x = side ? x1 : x0;
    ChunkWalk v = w;
    int64_t cut = w.total;
    if (c < w.shares && x < w.total) {
      const int owner = (int)place[2 * side];
      int64_t at = place[2 * side + 1];
      ChunkSeq q;
      if (w.cols > 1) {
        chunk_column(s, v, q, owner);
        for (int u = chunk_units(s, q, v.m); at + u <= x; u = chunk_units(s, q, v.m)) {
          at += u;
          chunk_skip(s, v, q, w.cols);
        }
        v.off = (int)(x - at);
      } else {
        for (v.b = owner * per;; ++v.b) {
          q = chunk_seq(s, v.b);
          if (q.n == 0) continue;
          const int64_t per_head = chunk_units_before(s, q, q.items);
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
      if (side == 0) { found[2] = v.b; found[3] = v.h; found[4] = v.m; found[5] = v.off; found[6] = v.col; }
    }
  }
  __syncthreads();
  w.pos = found[0]; w.end = found[1];
  w.b = (int)found[2]; w.h = (int)found[3]; w.m = (int)found[4]; w.off = (int)found[5]; w.col = (int)found[6];
  __syncthreads();
  return w;
}
#endif

}  // namespace earn

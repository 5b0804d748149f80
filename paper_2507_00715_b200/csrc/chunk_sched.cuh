// How the chunk attention deals its work to the CTAs, computed by every CTA from the device's lengths.
//
// A row tile holds the query rows (token, head) of `tile_tok` consecutive new tokens of one sequence under one head block (the
// query heads of a kv head, or a part of them where a group is larger than a tile).  A work item is `item_tok` tokens (one or
// two row tiles) against every key that its last token sees; its cost is counted in units, one per key tile.  The units of all
// items, in the order (sequence, head block, item, key tile), form one line, which is cut into equal shares, one per CTA: long
// lists are split over CTAs, short ones share one, whatever the mix of single tokens and long chunks.  A cut that falls close
// to an item's edge is moved there, so that only cuts that pay make partial results.  All of it is whole-number arithmetic on
// the lengths: every CTA finds its own share and, for an item in parts, who else holds one, without a planning kernel.
#pragma once
#include <stdint.h>

namespace earn {

struct ChunkSched {
  const int32_t* cu_new;    // [n_seq + 1] offsets of the sequences' new tokens
  const int32_t* seq_len;   // [n_seq] rows with the new ones
  int n_seq, n_tokens, max_len;
  int heads;                // head blocks: Hkv * ceil(g / heads of a block)
  int item_tok, key_tile;
  int grid, min_share;      // CTAs launched; units a CTA takes at least
};

struct ChunkSeq {
  int tok0, n, base;   // first new token, new tokens, rows in front of them (negative: the first new tokens have no row)
};
// Offsets that run past the batch or backwards are cut off, so that no row outside q and o is touched.
__host__ __device__ inline ChunkSeq chunk_seq(const ChunkSched& s, int b) {
  ChunkSeq q;
  int lo = s.cu_new[b], hi = s.cu_new[b + 1], len = s.seq_len[b];
  lo = lo < 0 ? 0 : lo > s.n_tokens ? s.n_tokens : lo;
  hi = hi < lo ? lo : hi > s.n_tokens ? s.n_tokens : hi;
  len = len < 0 ? 0 : len > s.max_len ? s.max_len : len;
  q.tok0 = lo; q.n = hi - lo; q.base = len - q.n;
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
// sum over i < n of floor((a i + b) / m), by the Euclidean recursion; a, b >= 0
__host__ __device__ inline int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
  int64_t sum = 0;
  while (true) {
    if (a >= m) { sum += (n - 1) * n / 2 * (a / m); a %= m; }
    if (b >= m) { sum += n * (b / m); b %= m; }
    const int64_t y = a * n + b;
    if (y < m) return sum;
    n = y / m;
    b = y % m;
    const int64_t t = m;
    m = a;
    a = t;
  }
}
// units of the first `count` items of a sequence under one head block
__host__ __device__ inline int64_t chunk_units_before(const ChunkSched& s, const ChunkSeq& q, int count) {
  const int items = (q.n + s.item_tok - 1) / s.item_tok;
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
    sum += floor_sum(whole - skip, s.key_tile, s.item_tok, (int64_t)q.base + (int64_t)(skip + 1) * s.item_tok + s.key_tile - 1);
  if (count >= items && items > 0) sum += chunk_units(s, q, items - 1);
  return sum;
}
__host__ __device__ inline int chunk_items(const ChunkSched& s, const ChunkSeq& q) { return (q.n + s.item_tok - 1) / s.item_tok; }

struct ChunkWalk {
  int64_t pos, end;    // units of the line: next one, and the end of this CTA's share
  int64_t total, tol;  // units in all; a cut closer than this to an item's edge is moved there
  int shares;          // shares the line is cut into
  int b, h, m, off;    // where pos is: unit `off` of item m under head block h of sequence b
  int longest;         // most new tokens of a sequence
};

__host__ __device__ inline int64_t chunk_cut(const ChunkWalk& w, int c) { return (int64_t)c * w.total / w.shares; }

// the item after (b, h, m): the same sequence's next one, the next head block, the next sequence with new tokens
__host__ __device__ inline void chunk_next(const ChunkSched& s, ChunkWalk& w, ChunkSeq& q) {
  w.off = 0;
  if (++w.m < chunk_items(s, q)) return;
  w.m = 0;
  if (++w.h < s.heads) return;
  w.h = 0;
  while (++w.b < s.n_seq) {
    q = chunk_seq(s, w.b);
    if (q.n > 0) return;
  }
}
// Finds unit x of the line, which lies `rem` units into sequence b (of `per_head` units per head block), and moves it to the
// item's edge where it is close to one.  Returns the cut; w receives the place if `place` is set.
__host__ __device__ inline int64_t chunk_settle(const ChunkSched& s, ChunkWalk& w, int64_t x, int b, ChunkSeq q, int64_t per_head,
                                                int64_t rem, bool place) {
  const int h = (int)(rem / per_head);
  const int64_t r = rem - (int64_t)h * per_head;
  int lo = 0, hi = chunk_items(s, q);   // the last item that starts at or before r
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (chunk_units_before(s, q, mid) <= r) lo = mid; else hi = mid;
  }
  const int off = (int)(r - chunk_units_before(s, q, lo)), left = chunk_units(s, q, lo) - off;
  const bool down = off <= w.tol, up = !down && left <= w.tol;
  if (place) {
    w.b = b; w.h = h; w.m = lo; w.off = down ? 0 : off;
    if (up) chunk_next(s, w, q);
  }
  return down ? x - off : up ? x + left : x;
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

#ifdef __CUDACC__
// This CTA's share of the line; every thread of the CTA calls it (`scratch`: shared memory for 64 64-bit words).
__device__ inline ChunkWalk chunk_share(const ChunkSched& s, int64_t* scratch) {
  const int t = threadIdx.x, threads = blockDim.x, lane = t & 31, warp = t >> 5;
  const int per = (s.n_seq + threads - 1) / threads, b0 = min(t * per, s.n_seq), b1 = min(b0 + per, s.n_seq);
  int64_t mine = 0;
  int longest = 0;
  for (int b = b0; b < b1; ++b) {
    const ChunkSeq q = chunk_seq(s, b);
    longest = max(longest, q.n);
    if (q.n > 0) mine += s.heads * chunk_units_before(s, q, chunk_items(s, q));
  }
  int64_t incl = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += v;
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 31) { scratch[warp] = incl; scratch[32 + warp] = longest; }
  __syncthreads();
  int64_t before = incl - mine, total = 0;
  for (int w = 0; w < threads / 32; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
    longest = max(longest, (int)scratch[32 + w]);
  }
  ChunkWalk w{};
  w.longest = longest;
  w.total = total;
  const int64_t shares = (total + s.min_share - 1) / s.min_share;
  w.shares = (int)(shares < s.grid ? (shares > 0 ? shares : 1) : s.grid);
  w.tol = total / w.shares / 16;
  const int c = blockIdx.x;
  __syncthreads();
  if (t == 0) {   // cuts at the line's ends, and CTAs without a share
    scratch[0] = 0; scratch[1] = c + 1 >= w.shares ? total : 0;
    scratch[2] = scratch[3] = scratch[4] = scratch[5] = 0;
    if (c >= w.shares) scratch[0] = total;
  }
  __syncthreads();
  if (c < w.shares && mine > 0) {
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      if (side == 1 && c + 1 >= w.shares) break;
      const int64_t x = chunk_cut(w, c + side);
      if (x < before || x >= before + mine) continue;
      int64_t at = before;
      for (int b = b0; b < b1; ++b) {
        const ChunkSeq q = chunk_seq(s, b);
        if (q.n == 0) continue;
        const int64_t per_head = chunk_units_before(s, q, chunk_items(s, q));
        if (x < at + s.heads * per_head) {
          scratch[side] = chunk_settle(s, w, x, b, q, per_head, x - at, side == 0);
          break;
        }
        at += s.heads * per_head;
      }
      if (side == 0) { scratch[2] = w.b; scratch[3] = w.h; scratch[4] = w.m; scratch[5] = w.off; }
    }
  }
  __syncthreads();
  w.pos = scratch[0]; w.end = scratch[1];
  w.b = (int)scratch[2]; w.h = (int)scratch[3]; w.m = (int)scratch[4]; w.off = (int)scratch[5];
  __syncthreads();
  return w;
}
#endif

}  // namespace earn

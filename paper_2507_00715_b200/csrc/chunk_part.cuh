// What the two chunk attention kernels for bf16 share: the parts of a CTA's share of the work, their hand-over, the joins of items
// that are cut, and the bounded waits between them.
#pragma once
#include "chunk_step.cuh"
#include "sm100_ptx.cuh"

namespace earn {
namespace {
using namespace ptx;

constexpr int BM = 128, BN = 128;                // rows of a row tile, keys of a key tile
constexpr long long WAIT_LIMIT = 2000000000LL;   // about one second of SM clocks

enum Form { PAIR, ROWS };                        // (of the tensor-core kernel)
enum Pass { FAST, MAXIMA, EXACT };

// One item's share of this CTA, as one warp hands it to the others (16 words in shared memory).
struct alignas(16) Part {
  int b, kvh, head0, n_heads;   // sequence, kv head, first query head, query heads
  int tok0, tok_in, n_tok;      // first token in the batch and in the chunk, tokens
  int base, keys;               // rows in front of the chunk; keys that the item's last token sees
  int u0, n;                    // key tiles u0 .. u0 + n - 1; n = 0: all parts have been handed out, n < 0: that was it
  int kind;                     // form, pass
  int n_rows;                   // rows of the first row tile
  int last;                     // the item's last key tile is among them
  int first, parts;             // CTAs first .. first + parts - 1 hold one part each
  __device__ __forceinline__ int pass() const { return kind >> 2; }
  __device__ __forceinline__ int form() const { return kind & 3; }
};
static_assert(sizeof(Part) == 64, "four 16-byte words");

// The CTA's parts one after the other; n = -1 behind the last.
__device__ __forceinline__ Part next_part(const ChunkArgs& a, const ChunkSched& s, ChunkWalk& w, ChunkSeq& q, int tile_tok, int pass) {
  Part p{};
  p.n = -1;
  if (w.pos >= w.end) return p;
  p.b = w.b;
  p.kvh = a.blocks > 1 ? w.h / a.blocks : w.h;
  p.head0 = p.kvh * a.g + (w.h - p.kvh * a.blocks) * a.block_heads;
  p.n_heads = min(a.block_heads, (p.kvh + 1) * a.g - p.head0);
  p.tok_in = w.m * s.item_tok;
  p.n_tok = min(s.item_tok, q.n - p.tok_in);
  p.tok0 = q.tok0 + p.tok_in;
  p.base = q.base;
  p.keys = chunk_keys(s, q, w.m);
  const int units = chunk_units(s, q, w.m);
  const int cost = chunk_cost(s, q, w.m), end = w.off + (int)min((uint32_t)(units - w.off), w.end - w.pos);
  p.u0 = max(w.off - cost, 0);
  p.n = end - cost - p.u0;
  p.n_rows = min(p.n_tok, tile_tok) * a.block_heads;
  p.kind = (p.n_tok > tile_tok ? PAIR : ROWS) + 4 * pass;
  p.last = end == units;
  p.parts = 1;
  if (w.off > 0 || !p.last) {
    const ChunkParts parts = chunk_parts(w, w.pos - w.off, units, cost);
    p.first = parts.first;
    p.parts = parts.parts;
  }
  w.pos += end - w.off;
  if (p.last) chunk_next(s, w, q);
  else w.off = end;
  return p;
}
// where this CTA's part of row tile x goes in the scratch
__device__ __forceinline__ int64_t part_slot(const Part& p, int x) {
  return (2 * (int64_t)blockIdx.x + ((int)blockIdx.x == p.first ? 1 : 0)) * 2 + x;
}

// The warp's arrival: what its lanes did before is visible to who waits.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
  __syncwarp();
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar) : "memory");
}
// Warp-wide bounded wait, the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, int parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, (uint32_t)parity & 1u, abort_flag, WAIT_LIMIT)) != 0;
}
// Part k in the ring of four places at `places`, from its warp; false: that was it, or a wait ran out.
__device__ __forceinline__ bool take_part(const void* places, uint32_t full, uint32_t free, int k, volatile int* abort_flag, Part& p) {
  const int at = k & 3;
  if (!warp_wait(full + 8u * at, k >> 2, abort_flag)) return false;
  const int4* from = reinterpret_cast<const int4*>(reinterpret_cast<const char*>(places) + at * 64);
  int4* to = reinterpret_cast<int4*>(&p);
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = from[i];
  warp_arrive(free + 8u * at);
  return p.n >= 0;
}
// Puts part `made` there; false: a wait ran out.
__device__ __forceinline__ bool give_part(void* places, uint32_t full, uint32_t free, int made, volatile int* abort_flag, const Part& p) {
  const int at = made & 3, lane = threadIdx.x & 31;
  if (made >= 4 && !warp_wait(free + 8u * at, (made >> 2) - 1, abort_flag)) return false;
  if (lane < 4)
    reinterpret_cast<int4*>(reinterpret_cast<char*>(places) + at * 64)[lane] =
        lane == 0 ? make_int4(p.b, p.kvh, p.head0, p.n_heads) : lane == 1 ? make_int4(p.tok0, p.tok_in, p.n_tok, p.base)
        : lane == 2 ? make_int4(p.keys, p.u0, p.n, p.kind) : make_int4(p.n_rows, p.last, p.first, p.parts);
  warp_arrive(full + 8u * at);
  return true;
}

// The CTA's n parts of items that are cut (at most its first part and its last) are written: joins those of which it was the last
// to finish.  (256 threads; x: row tile; flag: a word per part; weights: shared memory for 128 rows x 148 parts; sync: the threads' barrier, false if it gave up.)
template <int HD, bool ROW_MAJOR, class Sync>
__device__ __forceinline__ void join_cuts(const ChunkArgs& a, const Part* cuts, int n, int tile_tok, int x, int t, volatile int* flag, float* weights, Sync sync) {
  __threadfence();
  if (!sync()) return;
  if (t < n) {
    const Part& p = cuts[t];
    flag[t] = last_arrival(a.tickets + p.first * 2 + x, p.parts, a.status);
    __threadfence();
  }
  if (!sync()) return;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    if (flag[i] == 0) continue;
    const Part p = cuts[i];
    const int my_tok = p.form() == PAIR ? x * tile_tok : 0;
    ChunkParts parts;
    parts.first = p.first;
    parts.parts = p.parts;
    if (!sync()) return;   // (the weights before have been read)
    chunk_join<__nv_bfloat16, HD, BM, 256, true, ROW_MAJOR>(a, parts, 2, x, t, p.tok0 + my_tok, min(tile_tok, p.n_tok - my_tok), p.head0, p.n_heads, weights, sync);
  }
}

}  // namespace
}  // namespace earn

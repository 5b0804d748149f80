// Declarations of the calls of a step of several new tokens over a paged cache: page tables, rotary positions, chunk attention.
#pragma once
#include "chunk_sched.cuh"
#include "paged_cache.cuh"

namespace earn {

struct PageTableArgs {
  const int32_t* target;       // [n_seq] lengths to bring the sequences to
  const int32_t* held;         // [n_seq] rows held
  int32_t* held_out;           // may be held
  int32_t* block_table;        // [n_seq, pages_per_seq]
  int32_t* free_pages;         // [n_pages], a stack
  const int32_t* n_free;
  int32_t* n_free_out;         // may be n_free
  int32_t *cu_new, *seq_len, *positions, *slots, *n_refused;
  int32_t* ticket;
  int n_seq, n_tokens, pages_per_seq, n_pages;
};
constexpr int kPageTablesMaxSeqs = 16384;   // three numbers per sequence in shared memory
cudaError_t launch_page_tables(const PageTableArgs& a, cudaStream_t st);

struct RopeArgs {
  const char *q, *k, *v;       // rows of tokens `*_stride` bytes apart; heads follow one another; null: absent
  int64_t q_stride, k_stride, v_stride;
  char *q_out, *k_out;         // dense
  PagedSource cache;           // append form (k null otherwise): K and V rows go to slot slots[token]
  const int32_t *positions, *slots;
  const double* freq;          // radians per position of every pair
  int n_tokens, Hq, Hkv, D, dtype, rot, interleaved;
  float amplitude, sign;       // sign -1: the transposed rotation
};
cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st);

struct ChunkArgs {
  const void* q;
  void* o;
  float* lse;                  // [Hq, n_tokens] or null
  PagedSource cache;
  ChunkSched sched;
  float4* part_o;              // [2 * grid][row tiles][D / 4][rows], or [rows][D / 4]
  float2* part_ml;             // [2 * grid][row tiles][rows]: reference of the exponentials, their sum
  int32_t* tickets;            // [grid][row tiles], zero between calls
  int32_t* status;
  int Hq, Hkv, D, dtype, g;
  int block_heads, blocks;     // query heads of a head block, head blocks of a kv head
  float scale;
};
// Tiles that a call uses: rows of a row tile, row tiles of an item, keys of a key tile.
struct ChunkPlan {
  int rows, tiles, keys, block_heads, blocks, tile_tok, grid, min_share;
};
ChunkPlan plan_chunk_attn(int n_seq, int n_q_heads, int n_kv_heads, int D, int dtype, int n_tokens, int max_len);
cudaError_t launch_chunk_simt(const ChunkArgs& a, cudaStream_t st);                      // fp32
cudaError_t launch_chunk_tc(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st);    // bf16

// Softmax denominator of a row, natural log: once per row, so the logarithm is taken in 64 bits (the fast 32-bit one is off by
// a few 1e-7, which is all of what fp32 callers see).  A row that sees nothing: -inf.
template <bool LOG2>
__device__ __forceinline__ float chunk_lse(float ref, float sum) {
  if (sum == 0.f) return -INFINITY;
  return (float)((LOG2 ? (double)ref * 0.69314718055994530942 : (double)ref) + log((double)sum));
}

// Joins the parts of a row tile (all of them written, and seen by this thread) into its output rows: element (row, four
// columns) by element, `threads` threads of which this is number t.  The parts are added in their order along the keys, so
// the result does not depend on which of them came last.  LOG2: references are in the log2 domain, else natural.  ROW_MAJOR:
// a part is [rows][D], else [D / 4][rows][4].
template <typename T, int D, int ROWS, bool LOG2, bool ROW_MAJOR>
__device__ __forceinline__ void chunk_join(const ChunkArgs& a, const ChunkParts& parts, int tiles, int x, int t, int threads,
                                           int tok0, int n_tok, int head0, int n_heads) {
  constexpr int C4 = D / 4, AHEAD = 8;
  const int used = n_tok * a.block_heads;   // rows of the tile that hold a token
  for (int i = t; i < used * C4; i += threads) {
    const int row = ROW_MAJOR ? i / C4 : i % used, c4 = ROW_MAJOR ? i % C4 : i / used, tok = row / a.block_heads, head = row - tok * a.block_heads;
    if (head >= n_heads) continue;
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < parts.parts; p0 += AHEAD) {
      float2 ml[AHEAD];
      float4 v[AHEAD];
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        if (p0 + p >= parts.parts) { ml[p] = make_float2(-INFINITY, 0.f); v[p] = make_float4(0.f, 0.f, 0.f, 0.f); continue; }
        const int64_t slot = (int64_t)(2 * (parts.first + p0 + p) + (p0 + p == 0 ? 1 : 0)) * tiles + x;
        ml[p] = __ldcg(a.part_ml + slot * ROWS + row);
        v[p] = __ldcg(a.part_o + (ROW_MAJOR ? (slot * ROWS + row) * C4 + c4 : (slot * C4 + c4) * ROWS + row));
      }
      float mx = m;
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) mx = fmaxf(mx, ml[p].x);
      const float ref = mx == -INFINITY ? 0.f : mx;   // (nothing seen so far: every weight below is 2^-inf = 0)
      auto weight = [&](float from) { return LOG2 ? exp2f(from - ref) : exp2f((from - ref) * kLog2e); };
      const float keep = weight(m);
      l *= keep; acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const float w = weight(ml[p].x);
        l += ml[p].y * w;
        acc.x += v[p].x * w; acc.y += v[p].y * w; acc.z += v[p].z * w; acc.w += v[p].w * w;
      }
      m = mx;
    }
    const float inv = l == 0.f ? 0.f : __frcp_rn(l);
    const float y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
    Elem<T>::store4(reinterpret_cast<T*>(a.o) + ((int64_t)(tok0 + tok) * a.Hq + head0 + head) * D + c4 * 4, y);
    if (c4 == 0 && a.lse != nullptr)
      a.lse[(int64_t)(head0 + head) * a.sched.n_tokens + tok0 + tok] = chunk_lse<LOG2>(m, l);
  }
}

}  // namespace earn

// Declarations of the calls of a step of several new tokens over a paged cache: page tables, rotary positions, chunk attention.
#pragma once
#include "chunk_sched.cuh"
#include "paged_cache.cuh"
#include "sm100_ptx.cuh"

namespace earn {

// An arrival at a ticket that is zero between calls: true for the last of `all`, who sets it to zero again.  A ticket counts in steps
// of a large odd number, so that what other entry points leave in a workspace (counts, floats) is not taken for one of its states:
// whoever finds something else reports EARN_ERR_WORKSPACE.
constexpr uint32_t kTicketStep = 2654435769u, kTicketInverse = 340573321u;
static_assert(kTicketStep * kTicketInverse == 1u, "inverse modulo 2^32");
__device__ __forceinline__ bool last_arrival(int32_t* ticket, int all, int32_t* status) {
  const uint32_t before = (uint32_t)atomicAdd(ticket, (int32_t)kTicketStep) * kTicketInverse;
  if (before >= (uint32_t)all) atomicExch(status, (int32_t)EARN_ERR_WORKSPACE);
  if (before != (uint32_t)all - 1) return false;
  *ticket = 0;   // for the next call
  return true;
}

struct PageTableArgs {
  const int32_t* target;       // [n_seq] lengths to bring the sequences to
  const int32_t* held;         // [n_seq] rows held
  int32_t* held_out;           // may be held
  int32_t* block_table;        // [n_seq, pages_per_seq]
  int32_t* free_pages;         // [n_pages], a stack
  const int32_t* n_free;
  int32_t* n_free_out;         // may be n_free
  int32_t *cu_new, *seq_len, *positions, *slots, *n_refused;
  int32_t *ticket, *status;
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

constexpr int kChunkMaxLen = INT32_MAX - 127;   // the end of a list's last key tile is a 32-bit number
constexpr int kItemCost = 2;   // of the tensor-core kernel's items of two row tiles, see there
constexpr int kChunkTickets = 640;   // row tiles of all CTAs' items, at most

struct ChunkArgs {
  const void* q;
  void* o;
  float* lse;                  // [Hq, n_tokens] or null
  PagedSource cache;
  ChunkSched sched;
  ChunkSplit split;            // (bf16)
  float4* part_o;              // [2 * grid][row tiles][D / 4][rows], or [rows][D / 4]
  float2* part_ml;             // [2 * grid][row tiles][rows]: reference of the exponentials, their sum
  int32_t* tickets;            // [kChunkTickets >= grid * row tiles], zero between calls
  int32_t* status;
  int Hq, Hkv, D, dtype, g;
  int block_heads, blocks;     // query heads of a head block, head blocks of a kv head
  float scale;
};
// Tiles that a call uses: rows of a row tile, row tiles of an item, keys of a key tile.
struct ChunkPlan {
  int rows, tiles, keys, block_heads, blocks, tile_tok, grid, min_share;
  ChunkSplit split;            // (bf16)
};
ChunkPlan plan_chunk_attn(int n_seq, int n_q_heads, int n_kv_heads, int dtype, int n_tokens, int max_len);
cudaError_t launch_chunk_simt(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st);   // fp32
// bf16: the first kernel has items of 16 rows, which go through the keys one by one; the second fills row tiles of 128.  A call is
// the second's if it has items of several in a sequence and enough work for it (chunk_many; 24 units an SM: 256 rows over 2900, 8
// kv heads, 21 units: 46 and 62 us; 8 x 32 rows over 2900, 20 units: 49 and 48; 16 x 24 rows, 40 units: 87 and 72; one sequence of
// 128 rows over 9000, 2 kv heads, 8 units: 27 and 143; and at 16, 24, 32 and 40 units by their lists' length, 8 x 32 rows 41 and 44,
// 54 and 56, 65 and 67, 78 and 73; 8 x 96 rows 41 and 37, 55 and 39, 68 and 42, 81 and 41; one of 256 rows 40 and 59, 52 and 67, 63
// and 73, 75 and 73: level between 14 and 40 units, as the row tiles are filled).  The lengths are on the device, so both are launched, unless the sizes
// that the host knows tell, and one of them finds nothing to do, which costs 5 us.
cudaError_t launch_chunk_short(const ChunkArgs& a, cudaStream_t st);
cudaError_t launch_chunk_tc(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st);
constexpr int kShortRows = 16, kShortUnits = 24;   // rows of an item; units an SM, up to which a call is always the first kernel's

// Softmax denominator of a row, natural log: once per row, so the logarithm is taken in 64 bits (the fast 32-bit one is off by
// a few 1e-7, which is all of what fp32 callers see).  A row that sees nothing: -inf.
template <bool LOG2>
__device__ __forceinline__ float chunk_lse(float ref, float sum) {
  if (sum == 0.f) return -INFINITY;
  return (float)((LOG2 ? (double)ref * 0.69314718055994530942 : (double)ref) + log((double)sum));
}

// Joins the parts of a row tile (all of them written, and seen by this thread) into its output rows, by THREADS threads of
// which this is number t: first every part's weight in a row (2^(its reference - the largest) over the row's
// denominator, into `weights`, shared memory for used rows x parts numbers); then four columns of a row at a time.  The parts
// are added in their order along the keys, so the result does not depend on which of them came last.  LOG2: references are in the log2 domain, else natural.  ROW_MAJOR: a part is [rows][D], else
// [D / 4][rows][4].  sync(): barrier of the threads, false if it gave up.
template <typename T, int D, int ROWS, int THREADS, bool LOG2, bool ROW_MAJOR, class Sync>
__device__ __forceinline__ void chunk_join(const ChunkArgs& a, const ChunkParts& parts, int tiles, int x, int t,
                                           int tok0, int n_tok, int head0, int n_heads, float* weights, Sync sync) {
  constexpr int C4 = D / 4;
  const int used = n_tok * a.block_heads, n = parts.parts;   // rows of the tile that hold a token
  auto slot = [&](int p) { return (int64_t)(2 * (parts.first + p) + (p == 0 ? 1 : 0)) * tiles + x; };
  auto power = [&](float from, float ref) { return LOG2 ? exp2f(from - ref) : exp2f((from - ref) * kLog2e); };
  if constexpr (ROW_MAJOR) {
    // few rows: a lane per part, one trip to memory for all weights of a row (512 rows of one token: 11.9 -> 11.2 us; where a
    // part is a full row tile this code cost the kernel around it registers: 8 x 512 tokens of 64-wide heads 128 -> 136 us)
    const int lanes = n <= 4 ? 4 : 32, sub = t & (lanes - 1);
    const uint32_t mask = n <= 4 ? 0xfu << (t & 28) : 0xffffffffu;
    for (int row = t / lanes; row < used; row += THREADS / lanes) {
      const int tok = row / a.block_heads, head = row - tok * a.block_heads;
      if (head >= n_heads) continue;
      auto part = [&](int p) { return __ldcg(a.part_ml + slot(p) * ROWS + row); };
      const float2 mine = sub < n ? part(sub) : make_float2(-INFINITY, 0.f);
      float m = mine.x;
      for (int p = sub + lanes; p < n; p += lanes) m = fmaxf(m, part(p).x);
      for (int d = lanes / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(mask, m, d));
      const float ref = m == -INFINITY ? 0.f : m;   // (nothing seen: every weight is 2^-inf = 0)
      float l = mine.y * power(mine.x, ref);
      for (int p = sub + lanes; p < n; p += lanes) {
        const float2 ml = part(p);
        l += ml.y * power(ml.x, ref);
      }
      for (int d = lanes / 2; d > 0; d >>= 1) l += __shfl_xor_sync(mask, l, d);
      const float inv = l == 0.f ? 0.f : __frcp_rn(l);
      if (sub < n) weights[sub * used + row] = power(mine.x, ref) * inv;
      for (int p = sub + lanes; p < n; p += lanes) weights[p * used + row] = power(part(p).x, ref) * inv;
      if (sub == 0 && a.lse != nullptr) a.lse[(int64_t)(head0 + head) * a.sched.n_tokens + tok0 + tok] = chunk_lse<LOG2>(m, l);
    }
  } else {
    // a thread per row or, for many parts, a warp
    const bool by_warp = n > 4;
    const int lane = t & 31, lanes = by_warp ? 32 : 1;
    for (int row = by_warp ? t >> 5 : t; row < used; row += by_warp ? THREADS >> 5 : THREADS) {
      const int tok = row / a.block_heads, head = row - tok * a.block_heads;
      if (head >= n_heads) continue;
      float m = -INFINITY, l = 0.f;
#pragma unroll 4
      for (int p = by_warp ? lane : 0; p < n; p += lanes) m = fmaxf(m, __ldcg(a.part_ml + slot(p) * ROWS + row).x);
      if (by_warp) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      }
      const float ref = m == -INFINITY ? 0.f : m;   // (nothing seen: every weight is 2^-inf = 0)
#pragma unroll 4
      for (int p = by_warp ? lane : 0; p < n; p += lanes) {
        const float2 ml = __ldcg(a.part_ml + slot(p) * ROWS + row);
        l += ml.y * power(ml.x, ref);
      }
      if (by_warp) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
      }
      const float inv = l == 0.f ? 0.f : __frcp_rn(l);
#pragma unroll 4
      for (int p = by_warp ? lane : 0; p < n; p += lanes) weights[p * used + row] = power(__ldcg(a.part_ml + slot(p) * ROWS + row).x, ref) * inv;
      if ((!by_warp || lane == 0) && a.lse != nullptr) a.lse[(int64_t)(head0 + head) * a.sched.n_tokens + tok0 + tok] = chunk_lse<LOG2>(m, l);
    }
  }
  if (!sync()) return;
  if constexpr (!ROW_MAJOR) {
    // a thread has consecutive columns of one row, neighbouring threads neighbouring rows
    constexpr int PER = C4 * ROWS / THREADS, AHEAD = PER < 4 ? PER : 4;
    const int row = t % ROWS, from4 = t / ROWS * PER, tok = row / a.block_heads, head = row - tok * a.block_heads;
    if (row >= used || head >= n_heads) return;
    T* out = reinterpret_cast<T*>(a.o) + ((int64_t)(tok0 + tok) * a.Hq + head0 + head) * D;
#pragma unroll 1
    for (int c = from4; c < from4 + PER; c += AHEAD) {
      float4 acc[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
      for (int p = 0; p < n; ++p) {
        const float4* from = a.part_o + (slot(p) * C4 + c) * ROWS + row;
        const float w = weights[p * used + row];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const float4 v = __ldcg(from + k * ROWS);
          acc[k].x += v.x * w; acc[k].y += v.y * w; acc[k].z += v.z * w; acc[k].w += v.w * w;
        }
      }
      if constexpr (sizeof(T) == 2 && AHEAD % 2 == 0) {   // 16 bytes a store: neighbouring threads' rows are apart
#pragma unroll
        for (int k = 0; k < AHEAD; k += 2)
          *reinterpret_cast<uint4*>(out + (c + k) * 4) = make_uint4(ptx::pack_bf16(acc[k].x, acc[k].y), ptx::pack_bf16(acc[k].z, acc[k].w),
                                                                   ptx::pack_bf16(acc[k + 1].x, acc[k + 1].y), ptx::pack_bf16(acc[k + 1].z, acc[k + 1].w));
      } else {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const float y[4] = {acc[k].x, acc[k].y, acc[k].z, acc[k].w};
          Elem<T>::store4(out + (c + k) * 4, y);
        }
      }
    }
  } else {
    constexpr int BATCH = 2;   // elements of a thread in flight, four parts of each
    const int all = used * C4;
    for (int i0 = t; i0 < all; i0 += BATCH * THREADS) {
      float4 acc[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int p = 0; p < n; ++p) {
        const float4* from = a.part_o + slot(p) * ROWS * C4;
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const int i = i0 + k * THREADS;
          if (i >= all) continue;
          const float w = weights[p * used + i / C4];
          const float4 v = __ldcg(from + i);
          acc[k].x += v.x * w; acc[k].y += v.y * w; acc[k].z += v.z * w; acc[k].w += v.w * w;
        }
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int i = i0 + k * THREADS, row = i / C4, tok = row / a.block_heads, head = row - tok * a.block_heads;
        if (i >= all || head >= n_heads) continue;
        const float y[4] = {acc[k].x, acc[k].y, acc[k].z, acc[k].w};
        Elem<T>::store4(reinterpret_cast<T*>(a.o) + ((int64_t)(tok0 + tok) * a.Hq + head0 + head) * D + i % C4 * 4, y);
      }
    }
  }
}

}  // namespace earn

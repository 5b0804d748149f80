// Causal attention of every sequence's new tokens over its paged list, on the CUDA cores.
//
// fp32: products on the CUDA cores.  A CTA walks its share of the work (chunk_sched.cuh) item by item: 64 rows (token, head; 32 or
// 16 where there is less work than CTAs, or fewer rows in a sequence) against tiles of 64 keys, logits in registers (4 x 4 a
// thread), a running maximum and sum per row, probabilities through shared memory into the product with V.  Bound by the FMA
// pipes (2 x 1024 new tokens over 2000 rows, 12/2 heads: 30 TFLOP/s, half of what they can); few rows by shared memory reads.
#include <algorithm>

#include "chunk_step.cuh"

namespace earn {
namespace {

constexpr int KT = 64, THREADS = 256;

static_assert(2 * 320 <= kChunkTickets, "two row tiles a CTA");
constexpr int MAX_GRID = 320;   // CTAs, which is how many parts an item can have: the join wants a number per part and row
template <int D, int RT> constexpr int smem_floats() {
  constexpr int tiles = RT * D + 2 * KT * D + RT * KT;
  return tiles > MAX_GRID * RT ? tiles : MAX_GRID * RT;
}

template <typename T, int D, int RT>
__global__ void __launch_bounds__(THREADS) chunk_simt_kernel(ChunkArgs a) {
  constexpr int RI = RT / 16, DI = D / 64;
  extern __shared__ float4 smem4[];
  float* Qs = reinterpret_cast<float*>(smem4);
  float* Ks = Qs + RT * D;   // float4 c of row r lies at c ^ (r & 7): sixteen rows are read at once
  float* Vs = Ks + KT * D;
  float* Ps = Vs + KT * D;
  __shared__ int4 scratch[48];
  __shared__ int last_part;

  const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
  ChunkSched s = a.sched;
  pdl_launch_dependents();
  pdl_wait();
  ChunkWalk w = chunk_share(s, scratch, nullptr);
  if (w.pos >= w.end) return;
  ChunkSeq q = chunk_seq(s, w.b);
  while (w.pos < w.end) {
    const int units = chunk_units(s, q, w.m);
    const uint32_t start = w.pos - w.off;
    const int stop = (int)min((uint32_t)units, w.end - start);   // this part: units off .. stop
    const int kvh = w.h / a.blocks, head0 = kvh * a.g + (w.h % a.blocks) * a.block_heads;
    const int n_heads = min(a.block_heads, (kvh + 1) * a.g - head0);
    const int tok_in = w.m * s.item_tok, n_tok = min(s.item_tok, q.n - tok_in), tok0 = q.tok0 + tok_in;
    const int len = chunk_keys(s, q, w.m);
    __syncthreads();   // (the last item's reads of Qs are over)
    for (int i = t; i < RT * (D / 4); i += THREADS) {
      const int r = i / (D / 4), c = i % (D / 4), tok = r / a.block_heads, head = r % a.block_heads;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (tok < n_tok && head < n_heads)
        Elem<T>::load4(reinterpret_cast<const T*>(a.q) + ((int64_t)(tok0 + tok) * a.Hq + head0 + head) * D + c * 4, x);
      *reinterpret_cast<float4*>(Qs + r * D + c * 4) = make_float4(x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
    }
    int seen[RI];   // keys that the thread's rows see
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      const int tok = (ty * RI + i) / a.block_heads;
      seen[i] = tok < n_tok ? q.base + tok_in + tok + 1 : 0;
    }
    float m[RI], l[RI], acc[RI][DI * 4];
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
      for (int d = 0; d < DI * 4; ++d) acc[i][d] = 0.f;
    }
    for (int u = w.off; u < stop; ++u) {
      const int key0 = u * KT;
      __syncthreads();   // (reads of the last tiles are over)
      for (int i = t; i < KT * (D / 4); i += THREADS) {
        const int r = i / (D / 4), c = i % (D / 4);
        float kx[4] = {0.f, 0.f, 0.f, 0.f}, vx[4] = {0.f, 0.f, 0.f, 0.f};
        if (key0 + r < len) {
          bool named;
          const int page = paged_page(a.cache, w.b, (key0 + r) / EARN_PAGE_TOKENS, named);
          const int64_t at = (((int64_t)page * EARN_PAGE_TOKENS + (key0 + r) % EARN_PAGE_TOKENS) * a.Hkv + kvh) * D + c * 4;
          Elem<T>::load4(reinterpret_cast<const T*>(a.cache.k) + at, kx);
          Elem<T>::load4(reinterpret_cast<const T*>(a.cache.v) + at, vx);
        }
        *reinterpret_cast<float4*>(Ks + r * D + (c ^ (r & 7)) * 4) = make_float4(kx[0], kx[1], kx[2], kx[3]);
        *reinterpret_cast<float4*>(Vs + r * D + c * 4) = make_float4(vx[0], vx[1], vx[2], vx[3]);
      }
      __syncthreads();
      float x[RI][4];
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 4
      for (int c = 0; c < D / 4; ++c) {
        float4 kv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * j) * D + (c ^ (tx & 7)) * 4);
#pragma unroll
        for (int i = 0; i < RI; ++i) {
          const float4 qv = *reinterpret_cast<const float4*>(Qs + (ty * RI + i) * D + c * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[i][j] += qv.x * kv[j].x + qv.y * kv[j].y + qv.z * kv[j].z + qv.w * kv[j].w;
        }
      }
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (key0 + tx + 16 * j >= seen[i]) x[i][j] = -INFINITY;
          mx = fmaxf(mx, x[i][j]);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        mx = fmaxf(mx, m[i]);
        const float ref = mx == -INFINITY ? 0.f : mx;   // (nothing seen so far: every term is exp(-inf) = 0)
        const float keep = exp2f((m[i] - ref) * kLog2e);   // (subtracted in the natural domain: exact near the maximum)
        m[i] = mx;
        l[i] *= keep;
#pragma unroll
        for (int d = 0; d < DI * 4; ++d) acc[i][d] *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = exp2f((x[i][j] - ref) * kLog2e);
          l[i] += p;
          Ps[(ty * RI + i) * KT + tx + 16 * j] = p;
        }
      }
      __syncwarp();   // (a row's probabilities are written and read by the same half warp)
#pragma unroll 2
      for (int k4 = 0; k4 < KT / 4; ++k4) {
        float4 p[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) p[i] = *reinterpret_cast<const float4*>(Ps + (ty * RI + i) * KT + k4 * 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int d = 0; d < DI; ++d) {
            const float4 v = *reinterpret_cast<const float4*>(Vs + (k4 * 4 + k) * D + d * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < RI; ++i) {
              const float pk = k == 0 ? p[i].x : k == 1 ? p[i].y : k == 2 ? p[i].z : p[i].w;
              acc[i][d * 4 + 0] += pk * v.x; acc[i][d * 4 + 1] += pk * v.y;
              acc[i][d * 4 + 2] += pk * v.z; acc[i][d * 4 + 3] += pk * v.w;
            }
          }
        }
      }
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
    const ChunkParts parts = chunk_parts(w, start, units, 0);
    if (parts.parts == 1) {
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        const int row = ty * RI + i, tok = row / a.block_heads, head = row % a.block_heads;
        if (tok >= n_tok || head >= n_heads) continue;
        const float inv = l[i] == 0.f ? 0.f : __frcp_rn(l[i]);
#pragma unroll
        for (int d = 0; d < DI; ++d) {
          const float y[4] = {acc[i][d * 4] * inv, acc[i][d * 4 + 1] * inv, acc[i][d * 4 + 2] * inv, acc[i][d * 4 + 3] * inv};
          Elem<T>::store4(reinterpret_cast<T*>(a.o) + ((int64_t)(tok0 + tok) * a.Hq + head0 + head) * D + d * 64 + tx * 4, y);
        }
        if (tx == 0 && a.lse != nullptr)
          a.lse[(int64_t)(head0 + head) * s.n_tokens + tok0 + tok] = chunk_lse<false>(m[i], l[i]);
      }
    } else {
      const int64_t slot = 2 * (int64_t)blockIdx.x + ((int)blockIdx.x == parts.first ? 1 : 0);
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        const int row = ty * RI + i;
#pragma unroll
        for (int d = 0; d < DI; ++d)
          a.part_o[(slot * (D / 4) + d * 16 + tx) * RT + row] = make_float4(acc[i][d * 4], acc[i][d * 4 + 1], acc[i][d * 4 + 2], acc[i][d * 4 + 3]);
        if (tx == 0) a.part_ml[slot * RT + row] = make_float2(m[i], l[i]);
      }
      __threadfence();
      __syncthreads();
      if (t == 0) {
        last_part = last_arrival(a.tickets + parts.first, parts.parts, a.status);
        __threadfence();
      }
      __syncthreads();
      if (last_part) chunk_join<T, D, RT, THREADS, false, false>(a, parts, 1, 0, t, tok0, n_tok, head0, n_heads, Qs, [] { __syncthreads(); return true; });   // (in the tiles' memory)
    }
    w.pos += stop - w.off;
    if (stop == units) chunk_next(s, w, q);
    else w.off = stop;
  }
}

template <int D, int RT>
cudaError_t launch(const ChunkArgs& a, cudaStream_t st) {
  constexpr int bytes = smem_floats<D, RT>() * 4;
  cudaError_t e = ensure_dynamic_smem<chunk_simt_kernel<float, D, RT>>(bytes);
  if (e == cudaSuccess) e = launch_pdl(chunk_simt_kernel<float, D, RT>, dim3(a.sched.grid), dim3(THREADS), bytes, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}
template <int D>
cudaError_t launch_rows(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st) {
  return p.rows == 64 ? launch<D, 64>(a, st) : p.rows == 32 ? launch<D, 32>(a, st) : launch<D, 16>(a, st);
}

}  // namespace

ChunkPlan plan_chunk_attn(int n_seq, int n_q_heads, int n_kv_heads, int dtype, int n_tokens, int max_len) {
  ChunkPlan p{};
  const bool tc = dtype == EARN_BF16;
  p.rows = tc ? 128 : 64;
  p.tiles = tc ? 2 : 1;
  p.keys = tc ? 128 : KT;
  p.min_share = tc ? 2 : 1;
  const int g = n_q_heads / n_kv_heads;
  if (!tc) {
    // the largest row tile that is not twice the rows of an average sequence and leaves two units for every CTA (2 prompts of
    // 90-156 new tokens, 4 heads: 31 us with 64 rows, 19 with 16; 16 single tokens over 2000 rows: 93 and 62 us)
    const int64_t rows = std::max<int64_t>((int64_t)n_tokens * g / std::max(std::min(n_seq, n_tokens), 1), 1);
    auto work = [&](int r) { return (rows + r - 1) / r * std::min(n_seq, n_tokens) * n_kv_heads * ((max_len + KT - 1) / KT); };
    while (p.rows > 16 && (p.rows >= 2 * rows || work(p.rows) < 4 * sm_count())) p.rows /= 2;
  }
  p.blocks = (g + p.rows - 1) / p.rows;
  p.block_heads = (g + p.blocks - 1) / p.blocks;
  p.tile_tok = p.rows / p.block_heads;
  // no more CTAs than there can be units (bf16: of the kernel for few tokens, whose items are the smaller ones)
  const int blocks = tc ? (g + kShortRows - 1) / kShortRows : p.blocks, heads = (g + blocks - 1) / blocks, tokens = tc ? kShortRows / heads : p.tile_tok;
  const int64_t lists = std::min(n_seq, n_tokens), items = (int64_t)n_tokens / tokens + lists, tiles = (max_len + p.keys - 1) / p.keys;
  if (tc) {
    p.split.few = kShortRows / g;
    p.split.units = kShortUnits * sm_count() / (n_kv_heads * blocks);
    p.split.item_tok = tokens;
    p.split.known = n_tokens <= p.split.few || items * tiles <= p.split.units;
  }
  // Units are counted in 31 bits, by the kernel that works: for few tokens these are one item a list at most, or no more than
  // split.units.  (In floating point: the sizes' product may pass 64 bits.)
  const double units = (double)items * n_kv_heads * blocks * (tiles + (tc ? kItemCost : 0));
  const double counted = !tc ? units : p.split.known ? (double)lists * n_kv_heads * blocks * tiles
                         : (double)((int64_t)n_tokens / (p.tile_tok * p.tiles) + lists) * n_kv_heads * p.blocks * (tiles + kItemCost);
  const int most = std::min(tc ? sm_count() : 2 * sm_count(), MAX_GRID);
  p.grid = counted > (double)INT32_MAX ? 0 : units < most ? std::max((int)units, 1) : most;
  return p;
}

cudaError_t launch_chunk_simt(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st) {
  return a.D == 64 ? launch_rows<64>(a, p, st) : launch_rows<128>(a, p, st);
}

}  // namespace earn

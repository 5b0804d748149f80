// Causal attention over paged lists, for calls whose sequences have few new tokens each (decoded tokens, drafts) or that are too
// small to fill the GPU with row tiles: an item is 16 rows (token, query head of a kv head).
//
// Bound by HBM: every K and V row is read once for all rows, 2 D flop per byte and row, so the work is to keep the copies going.
// A CTA (one per SM) walks its share of the work line (chunk_sched.cuh).  One warp finds the parts and brings their tiles of 128
// keys, K and V, 64 KB a stage, three stages that run on across items: 128 to 192 KB are always on their way, more than the 60 KB
// that the SM's share of the bandwidth needs.  Eight warps have a page (16 keys) of every tile each and never wait for one
// another within an item: logits by mma.sync m16n8k16, a running maximum and sum per row, P V by the same instruction with P
// straight from the logits' registers.  When the item ends their outputs meet in shared memory.  (The tensor core's own
// instructions want 128 rows: the same calls on them, transposed to fill the rows with keys, spent most of their time in the
// waits between the product, the exponentials and the next product, with two such chains per SM: 84 us for 64 x 700-1044 rows.)
//
// The probabilities are rounded to bf16 for the product with V (chunk_tc.cu), their sum is that of the unrounded ones: the library's
// rule for bf16.  Two bf16 numbers per probability, measured: outputs off by 1.65e-3 of themselves, their own rounding, instead of
// 1.8e-3 to 2.4e-3, and 0.4 to 5 % more time (64 single tokens over 700-1044 rows 58.9 and 60.0 us, 32 rows over 9000 27.1 and 28.4).
//
// Measured: 64 single tokens over 700-1044 rows, 32/8 heads, 58 us (3.9 TB/s; 41 us of them the main loop); 8 over 20000-32000 rows
// 157 us (5.4 TB/s); 5 tokens over 2000 rows, 12/2 heads, 16 us.
//
// Every mbarrier wait is bounded, as in chunk_tc.cu.
#include <algorithm>

#include "chunk_part.cuh"
#include "mma_sync.cuh"
#include "tc_maps.cuh"

namespace earn {
namespace {

constexpr int WARPS = 8, THREADS = 32 * (WARPS + 1);
constexpr int NSTAGE = 3;

template <int HD>
struct Cfg {
  static constexpr int TILE = 128 * HD * 2, HALF = 128 * 128, NHALF = HD / 64;   // bytes of a tile, and of its 64-column blocks
  static constexpr int OFF_OUT = NSTAGE * 2 * TILE;                              // Q, later the warps' outputs, 16 KB
  static constexpr int OFF_SEQ = OFF_OUT + 16384, OFF_ML = OFF_SEQ + kChunkTable * (int)sizeof(ChunkSeq);   // [warp][row]
  static constexpr int ML_BYTES = WARPS * 16 * 8;
  static constexpr int OFF_PART = OFF_ML + ML_BYTES, OFF_CUT = OFF_PART + 4 * 64, OFF_BAR = OFF_CUT + 2 * 64;
  static constexpr int FULL = 0, EMPTY = FULL + NSTAGE, PARTFULL = EMPTY + NSTAGE, PARTFREE = PARTFULL + 4, GROUP = PARTFREE + 4, N_BARS = GROUP + 1;
  static constexpr int SMEM_BYTES = OFF_BAR + 8 * N_BARS + 32 + 1024;            // + alignment slack
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of an SM");
};

struct Consumer {
  uint8_t* gen;
  uint32_t base, bars;
  volatile int* abort_flag;
  int n_sync;
  template <class C>
  __device__ __forceinline__ bool sync() {   // the eight warps
    warp_arrive(bars + 8u * C::GROUP);
    return warp_wait(bars + 8u * C::GROUP, n_sync++, abort_flag);
  }
};

// The warps' outputs meet: R rows (of 16) x 512 / R columns at a time.  f: the lane's rows' factors.  out(row, column, y): two
// columns' sums, in the threads that hold them.
template <int HD, int R, class Out>
__device__ __forceinline__ bool exchange(Consumer& c, const float (&o)[HD / 8][4], const float (&f)[2], Out out) {
  using C = Cfg<HD>;
  constexpr int COLS = 512 / R < HD ? 512 / R : HD, PAIRS = COLS / 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = threadIdx.x;
  float2* all = reinterpret_cast<float2*>(c.gen + C::OFF_OUT);   // [warp][row][column pair], a row's pairs turned by four times its number
#pragma unroll
  for (int d0 = 0; d0 < HD; d0 += COLS) {
#pragma unroll
    for (int d = 0; d < COLS / 8; ++d) {
#pragma unroll
      for (int h = 0; h < (R > 8 ? 2 : 1); ++h) {
        const int r = h * 8 + (lane >> 2);
        if (R >= 8 || r < R)
          all[warp * 256 + r * PAIRS + ((d * 4 + (lane & 3) + 4 * r) & (PAIRS - 1))] = make_float2(o[d0 / 8 + d][h * 2] * f[h], o[d0 / 8 + d][h * 2 + 1] * f[h]);
      }
    }
    if (!c.template sync<C>()) return false;
    if (t < R * PAIRS) {
      const int r = t / PAIRS, pair = t % PAIRS;
      float2 y = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float2 v = all[i * 256 + r * PAIRS + ((pair + 4 * r) & (PAIRS - 1))];
        y.x += v.x;
        y.y += v.y;
      }
      out(r, d0 + pair * 2, y);
    }
    if (!c.template sync<C>()) return false;
  }
  return true;
}

// All parts of the CTA.
template <int HD>
__device__ __forceinline__ void consume(const ChunkArgs& a, Consumer c, float sl2) {
  using C = Cfg<HD>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = threadIdx.x;
  const uint32_t out = c.base + C::OFF_OUT;
  float2* ml = reinterpret_cast<float2*>(c.gen + C::OFF_ML);
  Part* cuts = reinterpret_cast<Part*>(c.gen + C::OFF_CUT);
  volatile int* flag = reinterpret_cast<volatile int*>(c.gen + C::OFF_BAR + 8 * C::N_BARS + 8);
  auto take = [&](int k, Part& p) { return take_part(c.gen + C::OFF_PART, c.bars + 8u * C::PARTFULL, c.bars + 8u * C::PARTFREE, k, c.abort_flag, p); };
  // Q: a thread brings 16 bytes of a row (shared memory: 128-byte lines of 64 columns, 16-byte chunk i of row r at i ^ (r % 8))
  const int q_row = t / (HD / 8), q_ch = t % (HD / 8), q_tok = q_row / a.block_heads, q_head = q_row - q_tok * a.block_heads;
  auto load_q = [&](const Part& p) {   // (rows that hold nothing are 0)
    uint4 v = make_uint4(0, 0, 0, 0);
    if (q_row < 16 && q_tok < p.n_tok && q_head < p.n_heads)
      v = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + ((int64_t)(p.tok0 + q_tok) * a.Hq + p.head0 + q_head) * HD + q_ch * 8);
    return v;
  };
  int n_cuts = 0, e = 0;   // ring entries taken so far
  Part p;
  bool more = take(0, p);
  if (!more) return;
  uint4 q_mine = load_q(p);
  for (int k = 0; more; ++k) {
    if (q_row < 16) st_shared_v4(out + (uint32_t)((q_ch >> 3) * (16 * 128) + q_row * 128 + (((q_ch & 7) ^ (q_row & 7)) << 4)), q_mine.x, q_mine.y, q_mine.z, q_mine.w);
    if (!c.template sync<C>()) return;
    uint32_t qf[HD / 16][4];
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
      const int r = lane & 15, ch = (kk & 3) * 2 + (lane >> 4);
      mma::ldsm_x4(out + (uint32_t)((kk >> 2) * (16 * 128) + r * 128 + ((ch ^ (r & 7)) << 4)), qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3]);
    }
    // a lane's rows: lane / 4 and 8 more; `seen`: keys that they see
    int seen[2];
    float m[2], l[2], o[HD / 8][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      seen[h] = p.base + p.tok_in + (h * 8 + (lane >> 2)) / a.block_heads + 1;
      m[h] = -INFINITY;
      l[h] = 0.f;
    }
#pragma unroll
    for (int d = 0; d < HD / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
    const int all_see = p.base + p.tok_in + 1;   // what every row sees
    for (int u = 0; u < p.n; ++u, ++e) {
      const int st = e % NSTAGE, key0 = (p.u0 + u) * BN + warp * EARN_PAGE_TOKENS;
      if (!warp_wait(c.bars + 8u * (C::FULL + st), e / NSTAGE, c.abort_flag)) return;
      const uint32_t sk = c.base + (uint32_t)(st * 2 * C::TILE), sv = sk + C::TILE;
      if (key0 < p.keys) {
        if (key0 + EARN_PAGE_TOKENS > p.keys) {   // rows behind the last key: a weight of zero does not undo a NaN
          const int from = p.keys - key0;
          for (int i = lane; i < (EARN_PAGE_TOKENS - from) * 8 * C::NHALF; i += 32) {
            const int r = from + (i >> 3) % (EARN_PAGE_TOKENS - from), h = (i >> 3) / (EARN_PAGE_TOKENS - from);
            st_shared_v4(sv + h * C::HALF + (warp * EARN_PAGE_TOKENS + r) * 128 + (i & 7) * 16, 0u, 0u, 0u, 0u);
          }
          fence_async_smem();   // (the stage's next copy comes behind these writes)
          __syncwarp();
        }
        float s[2][4], s1[2][4];   // (two chains of products each)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = s1[i >> 2][i & 3] = 0.f;
        const int kr = warp * EARN_PAGE_TOKENS + ((lane >> 4) << 3) + (lane & 7);   // K: matrices (keys 0-7, k 0-7), (0-7, 8-15), (8-15, 0-7), ..
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          uint32_t b[4];
          const int ch = (kk & 3) * 2 + ((lane >> 3) & 1);
          mma::ldsm_x4(sk + (kk >> 2) * C::HALF + kr * 128 + ((ch ^ (kr & 7)) << 4), b[0], b[1], b[2], b[3]);
          mma::mma_bf16((kk & 1) ? s1[0] : s[0], qf[kk], b[0], b[1]);
          mma::mma_bf16((kk & 1) ? s1[1] : s[1], qf[kk], b[2], b[3]);
        }
        float top[2];
        bool raise[2];
        const bool interior = key0 + EARN_PAGE_TOKENS <= all_see;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float mx = -INFINITY;
#pragma unroll
          for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float& x = s[n][h * 2 + i];
              x = interior || key0 + n * 8 + (lane & 3) * 2 + i < seen[h] ? (x + s1[n][h * 2 + i]) * sl2 : -INFINITY;
              mx = fmaxf(mx, x);
            }
          }
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          top[h] = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          raise[h] = top[h] > m[h] + 8.f || (m[h] == -INFINITY && top[h] > -INFINITY);
        }
        // A row's reference is raised when a logit exceeds it by more than 8 (no term exceeds 2^8): the first page as a rule.
        if (__any_sync(0xffffffffu, raise[0] || raise[1])) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float alpha = raise[h] ? ex2(m[h] - top[h]) : 1.f;
            if (raise[h]) m[h] = top[h];
            l[h] *= alpha;
#pragma unroll
            for (int d = 0; d < HD / 8; ++d) { o[d][h * 2] *= alpha; o[d][h * 2 + 1] *= alpha; }
          }
        }
        uint32_t pf[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float ref = m[h] == -INFINITY ? 0.f : m[h];   // (nothing seen so far: every term is 2^-inf = 0)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float p0 = ex2(s[n][h * 2] - ref), p1 = ex2(s[n][h * 2 + 1] - ref);
            l[h] += p0 + p1;
            pf[n * 2 + h] = pack_bf16(p0, p1);
          }
        }
        const int vr = warp * EARN_PAGE_TOKENS + (((lane >> 3) & 1) << 3) + (lane & 7);   // V: matrices (keys 0-7, d 0-7), (8-15, 0-7), (0-7, 8-15), ..
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          uint32_t b[4];
          const int ch = (d & 3) * 2 + (lane >> 4);
          mma::ldsm_x4_t(sv + (d >> 2) * C::HALF + vr * 128 + ((ch ^ (vr & 7)) << 4), b[0], b[1], b[2], b[3]);
          mma::mma_bf16(o[2 * d], pf, b[0], b[1]);
          mma::mma_bf16(o[2 * d + 1], pf, b[2], b[3]);
        }
      }
      warp_arrive(c.bars + 8u * (C::EMPTY + st));
    }
    // ---- the warps' sums and references meet, then their outputs; the next part's Q is on its way meanwhile
    Part next;
    more = take(k + 1, next);
    if (more) q_mine = load_q(next);
    const bool whole = p.parts == 1;
    const int64_t slot = part_slot(p, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      if ((lane & 3) == 0) ml[warp * 16 + h * 8 + (lane >> 2)] = make_float2(m[h], l[h]);
    }
    if (!c.template sync<C>()) return;   // (and Q has been read)
    // the lane's rows' factors, 2^(reference - the warps' largest) over the denominator
    float f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = h * 8 + (lane >> 2);
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) mx = fmaxf(mx, ml[i * 16 + row].x);
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float2 v = ml[i * 16 + row];
        sum += v.y * ex2(v.x - ref);
      }
      f[h] = ex2(m[h] - ref);
      if (whole) f[h] *= sum == 0.f ? 0.f : __frcp_rn(sum);
      const int tok = row / a.block_heads, head = row - tok * a.block_heads;
      if (warp == 0 && (lane & 3) == 0 && tok < p.n_tok && head < p.n_heads) {
        if (!whole) a.part_ml[slot * BM + row] = make_float2(mx, sum);
        else if (a.lse != nullptr) a.lse[(int64_t)(p.head0 + head) * a.sched.n_tokens + p.tok0 + tok] = chunk_lse<true>(mx, sum);
      }
    }
    auto store = [&](int row, int col, float2 y) {
      const int tok = row / a.block_heads, head = row - tok * a.block_heads;
      if (tok >= p.n_tok || head >= p.n_heads) return;
      if (whole)
        *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(a.o) + ((int64_t)(p.tok0 + tok) * a.Hq + p.head0 + head) * HD + col) = pack_bf16(y.x, y.y);
      else
        *reinterpret_cast<float2*>(reinterpret_cast<float*>(a.part_o) + (slot * BM + row) * HD + col) = y;
    };
    const int used = p.n_tok * a.block_heads;
    const bool met = used <= 4 ? exchange<HD, 4>(c, o, f, store) : used <= 8 ? exchange<HD, 8>(c, o, f, store) : exchange<HD, 16>(c, o, f, store);
    if (!met) return;
    if (!whole) {
      if (t == 0) cuts[n_cuts] = p;
      ++n_cuts;
    }
    p = next;
  }
  if (*c.abort_flag == 0 && n_cuts > 0)   // (the ring's memory holds the weights: nothing is on its way any more)
    join_cuts<HD, true>(a, cuts, n_cuts, a.sched.item_tok, 0, t, flag, reinterpret_cast<float*>(c.gen), [&]() { return c.template sync<C>(); });
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
chunk_short_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ChunkArgs a, float sl2) {
  using C = Cfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;    // swizzled tiles need 1024-byte alignment
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + C::OFF_BAR;
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + C::OFF_BAR + 8 * C::N_BARS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSTAGE; ++i) {
      mbar_init(bar(C::FULL + i), 1);
      mbar_init(bar(C::EMPTY + i), WARPS);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(C::PARTFULL + i), 1);
      mbar_init(bar(C::PARTFREE + i), WARPS);
    }
    mbar_init(bar(C::GROUP), WARPS);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  if (chunk_many(a.sched, a.split)) return;   // (the call is the other kernel's)
  ChunkSched sched = a.sched;
  ChunkWalk w = chunk_share(sched, reinterpret_cast<int4*>(gen), reinterpret_cast<ChunkSeq*>(gen + C::OFF_SEQ));
  if (w.pos >= w.end) return;   // (the same for all threads)
  fence_async_smem();           // (the copies that come next land where the shares' scratch was)
  __syncthreads();
  if (warp == WARPS) {
    // ------------------------------------------------------------------ parts, and the copies of their pages
    ChunkSeq q = chunk_seq(sched, w.b);
    int e = 0;
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const Part p = next_part(a, sched, w, q, sched.item_tok, FAST);
      ok = give_part(gen + C::OFF_PART, bar(C::PARTFULL), bar(C::PARTFREE), k, abort_flag, p);
      if (!ok || p.n < 0) break;
      const int n_pages = (p.keys + EARN_PAGE_TOKENS - 1) / EARN_PAGE_TOKENS;
      const int pg = lane & 7, half = (lane >> 3) % C::NHALF, is_v = (lane >> 3) / C::NHALF;   // a lane's page, 64-column block, K or V
      bool named = false;
      int next_page = pg < n_pages - p.u0 * 8 ? paged_page(a.cache, p.b, p.u0 * 8 + pg, named) : 0;
      for (int u = 0; u < p.n; ++u, ++e) {
        const int st = e % NSTAGE, pages = min(n_pages - (p.u0 + u) * 8, 8), page = next_page;
        if (u + 1 < p.n && pg < n_pages - (p.u0 + u + 1) * 8) next_page = paged_page(a.cache, p.b, (p.u0 + u + 1) * 8 + pg, named);   // (in flight meanwhile)
        if (e >= NSTAGE && !warp_wait(bar(C::EMPTY + st), (e / NSTAGE) - 1, abort_flag)) { ok = false; break; }
        if (lane == 0) mbar_expect_tx(bar(C::FULL + st), (uint32_t)max(pages, 0) * (2 * EARN_PAGE_TOKENS * HD * 2));
        __syncwarp();
        if (pg < pages && is_v < 2)
          tma_load_3d(base + (uint32_t)(st * 2 * C::TILE + is_v * C::TILE + half * C::HALF + pg * (EARN_PAGE_TOKENS * 128)), is_v ? &map_v : &map_k,
                      bar(C::FULL + st), half * 64, p.kvh, page * EARN_PAGE_TOKENS);
      }
    }
    if (*abort_flag) {
      int none = 0;
      for (int f = max(e - NSTAGE, 0); f < e; ++f) mbar_wait_bounded(bar(C::FULL + f % NSTAGE), (f / NSTAGE) & 1, &none, WAIT_LIMIT);
    }
  } else {
    Consumer c{gen, base, bars, abort_flag, 0};
    consume<HD>(a, c, sl2);
  }
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, (int32_t)EARN_ERR_TIMEOUT);
}

template <int HD>
cudaError_t launch(const ChunkArgs& a, cudaStream_t st) {
  CUtensorMap mk, mv;
  const int rows = a.cache.n_pages * EARN_PAGE_TOKENS;
  if (!tcmap::make_map(&mk, a.cache.k, a.Hkv, rows, EARN_PAGE_TOKENS, HD) || !tcmap::make_map(&mv, a.cache.v, a.Hkv, rows, EARN_PAGE_TOKENS, HD))
    return cudaErrorInvalidValue;
  ChunkArgs s = a;
  s.blocks = (a.g + kShortRows - 1) / kShortRows;   // head blocks of at most 16 heads
  s.block_heads = (a.g + s.blocks - 1) / s.blocks;
  s.sched.heads = a.Hkv * s.blocks;
  s.sched.item_tok = a.split.item_tok;
  s.sched.min_share = 1;
  cudaError_t e = ensure_dynamic_smem<chunk_short_kernel<HD>>(Cfg<HD>::SMEM_BYTES);
  if (e == cudaSuccess)
    e = launch_pdl(chunk_short_kernel<HD>, dim3(s.sched.grid), dim3(THREADS), Cfg<HD>::SMEM_BYTES, st, mk, mv, s, a.scale * kLog2e);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_chunk_short(const ChunkArgs& a, cudaStream_t st) { return a.D == 64 ? launch<64>(a, st) : launch<128>(a, st); }

}  // namespace earn

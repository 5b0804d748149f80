// One new token per sequence over the paged cache of a full layer (Eq. 4: append K_t, V_t, then attend over K_{1:t}), with
// the attention weight every row received added to its accumulated weight.
//
// HBM-bound: K and V of every row are read once for every 16 query heads of a kv head.  The key list of a (sequence, kv head) is cut into chunks; a warp takes
// one chunk under 16 query rows (the group's heads), page by page -- a page is a tile of 16 positions -- through a ring
// of cp.async stages, and leaves a normalised partial with its log2-domain softmax denominator.  A second kernel joins
// the partials.  The weight of a row needs the denominator of the whole list, so the first kernel also leaves the scaled
// logits (4 bytes per query head and row beside the 4 D bytes of K and V: 6 % at a group of 8 and D = 128; where a call's
// logits outgrow L2 beside its K and V they go through DRAM, 35 MB written and 52 MB read over 8 lists of 20000 to 32768 rows
// in a cold-cache profile), and the second kernel turns them into weights: sum over the heads of 2^(logit - LSE).
// 32/8 heads of 128, with weights: 168 us over 8 lists of 20000 to 32768 rows (5.4 TB/s, 0.84 of a copy; the first kernel
// alone 151 us), 51 us over 64 of 700 to 1044 (44 us alone).  The last warp of a (sequence, kv head) joining by itself
// instead of a second kernel cost 66 us there: one warp is too few for the logits.
// (Times in this file are of calls replayed from a graph; issued one by one the two above take 173 and 52 us.)
// Small calls: one launch, the chunks of a list in a cluster (below).
// No atomics: every sum has one order.
#include <cfloat>
#include <climits>
#include <type_traits>

#include "decode_tile.cuh"
#include "paged_cache.cuh"
#include "sm100_ptx.cuh"

namespace earn {
namespace {
using namespace dec;

constexpr int STAGES = 4;

// One warp's 16 query rows against tiles of 16 or 32 positions, as RowTile, with the logits of every tile handed on:
// sink(at, fragments) receives the (masked, unscaled) logits of the 8-column blocks that start at tile `at`.
// The probabilities are rounded to bf16 in front of V, as in the other decode kernels: the output is off by 1.93e-3 of itself
// (root of the mean square, 64 lists of 700 to 1044 rows) where the output's own rounding is 1.66e-3.  Two bf16 numbers
// per probability and twice the products with V would leave that alone, for 1 to 8 % more time (64 lists 51.0 -> 52.6 us, one 5.7
// -> 6.1, group of 7 33.6 -> 35.6).
template <int D>
struct PagedTile : RowTile<D> {
  using Base = RowTile<D>;
  using Base::KSTEPS;
  using Base::NTILES;
  using Base::l0;
  using Base::l1;
  using Base::m0;
  using Base::m1;
  using Base::o;
  using Base::qf;

  // One tile of KT positions: S = Q K^T, online softmax, O += P V.  ks / vs: shared-memory addresses of the K and V
  // tiles.  When `masked`, visible(column, second_row) says whether position `column` of the tile counts for the
  // lane's first (false) or second (true) row.
  template <typename Vis, typename Sink>
  __device__ __forceinline__ void attend(uint32_t ks, uint32_t vs, float scale_log2, int lane, bool masked, Vis visible,
                                         Sink sink, int at) {
    constexpr int PITCH = Geo<D>::PITCH;
    const int c2 = (lane & 3) * 2, mat = lane >> 3;
    const uint32_t k_lane = (uint32_t)(((mat >> 1) << 3) + (lane & 7)) * PITCH + (uint32_t)(mat & 1) * 16;
    const uint32_t v_lane = (uint32_t)(((mat & 1) << 3) + (lane & 7)) * PITCH + (uint32_t)(mat >> 1) * 16;
    // two accumulator sets per 8-column block (even / odd k-steps) halve the chain of dependent MMAs
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, s2[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk += 2) {
      uint32_t b0, b1, b2, b3, c0, c1, c2_, c3;
      ldsm_x4(ks + k_lane + kk * 32, b0, b1, b2, b3);
      ldsm_x4(ks + k_lane + (kk + 1) * 32, c0, c1, c2_, c3);
      mma_bf16(s[0], qf[kk], b0, b1);
      mma_bf16(s[1], qf[kk], b2, b3);
      mma_bf16(s2[0], qf[kk + 1], c0, c1);
      mma_bf16(s2[1], qf[kk + 1], c2_, c3);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] += s2[n][e];
    if (masked) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!visible(n * 8 + c2 + (e & 1), e >= 2)) s[n][e] = -INFINITY;
    }
    sink(at, s);
    float mx0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
    float mx1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
    const float mn0 = fmaxf(m0, mx0 * scale_log2), mn1 = fmaxf(m1, mx1 * scale_log2);
    const float al0 = ex2(m0 - mn0), al1 = ex2(m1 - mn1);
    const bool grew = (mn0 != m0) || (mn1 != m1);
    m0 = mn0;
    m1 = mn1;
    uint32_t pf[4];
    {
      float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float p0 = ex2(fmaf(s[n][0], scale_log2, -mn0)), p1 = ex2(fmaf(s[n][1], scale_log2, -mn0));
        const float p2 = ex2(fmaf(s[n][2], scale_log2, -mn1)), p3 = ex2(fmaf(s[n][3], scale_log2, -mn1));
        sum0 += p0 + p1;
        sum1 += p2 + p3;
        pf[n * 2] = pack2(p0, p1);
        pf[n * 2 + 1] = pack2(p2, p3);
      }
      l0 = l0 * al0 + sum0;   // per-lane partial sums; reduced over the quad by finish()
      l1 = l1 * al1 + sum1;
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NTILES; ++n) { o[n][0] *= al0; o[n][1] *= al0; o[n][2] *= al1; o[n][3] *= al1; }
    }
#pragma unroll
    for (int nn = 0; nn < NTILES / 2; ++nn) {
      uint32_t b0, b1, b2, b3;
      ldsm_x4_t(vs + v_lane + nn * 32, b0, b1, b2, b3);
      mma_bf16(o[2 * nn], pf, b0, b1);
      mma_bf16(o[2 * nn + 1], pf, b2, b3);
    }
  }

  // Two whole tiles (2 * KT positions, every one visible to every row) in one softmax step: four independent chains
  // of MMAs instead of two, one rescale of the accumulator and one round of quad shuffles per 32 positions.
  template <typename Sink>
  __device__ __forceinline__ void attend2(uint32_t ksa, uint32_t vsa, uint32_t ksb, uint32_t vsb, float scale_log2, int lane,
                                          Sink sink, int at) {
    constexpr int PITCH = Geo<D>::PITCH;
    const int mat = lane >> 3;
    const uint32_t k_lane = (uint32_t)(((mat >> 1) << 3) + (lane & 7)) * PITCH + (uint32_t)(mat & 1) * 16;
    const uint32_t v_lane = (uint32_t)(((mat & 1) << 3) + (lane & 7)) * PITCH + (uint32_t)(mat >> 1) * 16;
    float s[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) {
      uint32_t b0, b1, b2, b3, c0, c1, c2_, c3;
      ldsm_x4(ksa + k_lane + kk * 32, b0, b1, b2, b3);
      ldsm_x4(ksb + k_lane + kk * 32, c0, c1, c2_, c3);
      mma_bf16(s[0], qf[kk], b0, b1);
      mma_bf16(s[1], qf[kk], b2, b3);
      mma_bf16(s[2], qf[kk], c0, c1);
      mma_bf16(s[3], qf[kk], c2_, c3);
    }
    sink(at, s);
    float mx0 = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), fmaxf(fmaxf(s[2][0], s[2][1]), fmaxf(s[3][0], s[3][1])));
    float mx1 = fmaxf(fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3])), fmaxf(fmaxf(s[2][2], s[2][3]), fmaxf(s[3][2], s[3][3])));
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
    const float mn0 = fmaxf(m0, mx0 * scale_log2), mn1 = fmaxf(m1, mx1 * scale_log2);
    const float al0 = ex2(m0 - mn0), al1 = ex2(m1 - mn1);
    const bool grew = (mn0 != m0) || (mn1 != m1);
    m0 = mn0;
    m1 = mn1;
    uint32_t pf[2][4];
    {
      float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float p0 = ex2(fmaf(s[n][0], scale_log2, -mn0)), p1 = ex2(fmaf(s[n][1], scale_log2, -mn0));
        const float p2 = ex2(fmaf(s[n][2], scale_log2, -mn1)), p3 = ex2(fmaf(s[n][3], scale_log2, -mn1));
        sum0 += p0 + p1;
        sum1 += p2 + p3;
        pf[n >> 1][(n & 1) * 2] = pack2(p0, p1);
        pf[n >> 1][(n & 1) * 2 + 1] = pack2(p2, p3);
      }
      l0 = l0 * al0 + sum0;
      l1 = l1 * al1 + sum1;
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NTILES; ++n) { o[n][0] *= al0; o[n][1] *= al0; o[n][2] *= al1; o[n][3] *= al1; }
    }
#pragma unroll
    for (int nn = 0; nn < NTILES / 2; ++nn) {
      uint32_t b0, b1, b2, b3, c0, c1, c2_, c3;
      ldsm_x4_t(vsa + v_lane + nn * 32, b0, b1, b2, b3);
      ldsm_x4_t(vsb + v_lane + nn * 32, c0, c1, c2_, c3);
      mma_bf16(o[2 * nn], pf[0], b0, b1);
      mma_bf16(o[2 * nn + 1], pf[0], b2, b3);
      mma_bf16(o[2 * nn], pf[1], c0, c1);
      mma_bf16(o[2 * nn + 1], pf[1], c2_, c3);
    }
  }
};

// four rows' weights: out[0..3] = before + w for the rows j + i < n; row `fresh` (the appended one, or outside) starts from zero
__device__ __forceinline__ void add_weights(float* out, const float4& before, int j, int n, int fresh, const float (&w)[4]) {
  const float x[4] = {(fresh == j ? 0.f : before.x) + w[0], (fresh == j + 1 ? 0.f : before.y) + w[1],
                      (fresh == j + 2 ? 0.f : before.z) + w[2], (fresh == j + 3 ? 0.f : before.w) + w[3]};
  if (j + 4 <= n) {
    *reinterpret_cast<float4*>(out) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < n) out[i] = x[i];
  }
}

// ------------------------------------------------------------------------------------------------ thread-block clusters
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// address of the same shared-memory location in CTA `rank` of the cluster, and loads from there
__device__ __forceinline__ uint32_t peer_smem(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float peer_ld(uint32_t addr) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
  return x;
}
__device__ __forceinline__ float4 peer_ld4(uint32_t addr) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
  return x;
}

// ------------------------------------------------------------------------------------------------ bf16: one warp per chunk
// CLUSTER: the list of a (sequence, kv head) is shared out to the one-warp CTAs of a cluster (a.cluster of them, at most 512
// rows each).  Logits stay in shared memory, the CTAs read each other's maxima, sums and partial rows through distributed
// shared memory, and each finishes its share of the output and the weights of its rows: one launch, nothing through L2.
// Behind the ring: logits [g][chunk + 8] (with weights), maxima and sums [2][16], what a CTA's partial counts [8][16], LSE [16].
constexpr int kMaxCluster = 8;
template <int D>
__host__ __device__ constexpr int cluster_smem(int g, int chunk, bool weigh) {
  return STAGES * Geo<D>::STAGE_B + (weigh ? g * (chunk + 8) * 4 : 0) + (2 + kMaxCluster + 1) * 16 * 4;
}

template <int D, bool WEIGH, bool CLUSTER>
__global__ void __launch_bounds__(32) paged_decode_kernel(PagedDecodeArgs a) {
  using G = Geo<D>;
  constexpr int CH = G::CH, RPI = G::RPI, NIT = KT / RPI, NTILES = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  pdl_wait();
  const int lane = threadIdx.x;
  const int row_tiles = (a.g + 15) / 16;
  const int kvh = CLUSTER ? blockIdx.x / a.cluster : blockIdx.x, b = blockIdx.z;
  const int split = CLUSTER ? (int)cluster_rank() : (int)blockIdx.y / row_tiles, row0 = CLUSTER ? 0 : (blockIdx.y % row_tiles) * 16;
  const int len = paged_len(a.cache, b);
  const int chunk = CLUSTER ? ((len + KT - 1) / KT + a.cluster - 1) / a.cluster * KT : a.chunk;   // rows of a CTA
  const int begin = split * chunk, n = min(len - begin, chunk);
  if (!CLUSTER && n <= 0) return;
  const int n_tiles = (n + KT - 1) / KT;
  const float scale_log2 = a.scale * kLog2e;
  RowMap rm;
  rm.b = b; rm.kvh = kvh; rm.row0 = row0; rm.g = a.g; rm.W = 1; rm.n_rows = a.g; rm.Hq = a.Hq;
  const bf16 *kp = reinterpret_cast<const bf16*>(a.cache.k), *vp = reinterpret_cast<const bf16*>(a.cache.v);
  const bf16 *kn = reinterpret_cast<const bf16*>(a.k_new), *vn = reinterpret_cast<const bf16*>(a.v_new);

  // lane t holds the page of tile t (a chunk has at most 32 tiles)
  bool page_ok = true;
  int page = 0;
  if (lane < n_tiles) page = paged_page(a.cache, b, begin / KT + lane, page_ok);

  const uint32_t ring = ptx::smem_u32(smem);
  const int ch = lane % CH, r0 = lane / CH;
  const uint32_t dst0 = (uint32_t)r0 * G::PITCH + (uint32_t)ch * 16;
  const int64_t rowstride = (int64_t)a.Hkv * D;
  const int newest = kn != nullptr ? len - 1 - begin : -1;   // position of the appended row in this chunk's list (or outside)
  const int64_t new_off = ((int64_t)b * a.Hkv + kvh) * D + ch * 8;

  auto issue_tile = [&](int t) {
    const int pg = __shfl_sync(0xffffffffu, page, t);
    const uint32_t kdst = ring + (t % STAGES) * G::STAGE_B + dst0, vdst = kdst + G::TILE_B;
    const int64_t off = (((int64_t)pg * KT + r0) * a.Hkv + kvh) * D + ch * 8;
    if ((t + 1) * KT <= n && (newest < t * KT || newest >= (t + 1) * KT)) {
#pragma unroll
      for (int i = 0; i < NIT; ++i) {
        cp_async16(kdst + i * RPI * G::PITCH, kp + off + i * RPI * rowstride);
        cp_async16(vdst + i * RPI * G::PITCH, vp + off + i * RPI * rowstride);
      }
    } else {   // rows past the list are zero-filled; the appended row comes from k_new / v_new
#pragma unroll
      for (int i = 0; i < NIT; ++i) {
        const int p = t * KT + r0 + i * RPI;
        const bool fresh = p == newest;
        const bf16* ks = fresh ? kn + new_off : kp + off + i * RPI * rowstride;
        const bf16* vs = fresh ? vn + new_off : vp + off + i * RPI * rowstride;
        cp_async16(kdst + i * RPI * G::PITCH, ks, p < n ? 16 : 0);
        cp_async16(vdst + i * RPI * G::PITCH, vs, p < n ? 16 : 0);
      }
    }
  };
  // tiles are consumed in pairs: two in use, STAGES - 2 in flight
  constexpr int PRE = STAGES - 2;
#pragma unroll
  for (int s = 0; s < PRE; ++s) {
    if (s < n_tiles) issue_tile(s);
    cp_async_commit();
  }
  PagedTile<D> t;
  t.init(reinterpret_cast<const bf16*>(a.q), rm, lane);
  t.m0 = t.m1 = -FLT_MAX;   // (a finite floor: rows whose logits are all -inf so far subtract to 2^-inf, not to NaN)

  // logits of tile `tile` (8-column blocks 0 .. NB - 1 from its first position on) -> scores, this lane's two rows
  const int q0 = row0 + (lane >> 2), q1 = q0 + 8, c2 = (lane & 3) * 2;
  float* s_base = !WEIGH ? nullptr : CLUSTER ? reinterpret_cast<float*>(smem + STAGES * G::STAGE_B)
                                             : a.scores + ((int64_t)b * a.Hkv + kvh) * a.g * a.score_ld + begin;
  const int64_t s_ld = CLUSTER ? chunk + 8 : a.score_ld;   // (+ 8: the rows of a fragment's store fall into different banks)
  auto store = [&](int tile, const float* s0, int blk) {   // s0: the four fragment values of 8-column block blk
    if (!WEIGH) return;
    const int c = tile * KT + blk * 8 + c2;
    if (q0 < a.g) *reinterpret_cast<float2*>(s_base + q0 * s_ld + c) = make_float2(s0[0] * scale_log2, s0[1] * scale_log2);
    if (q1 < a.g) *reinterpret_cast<float2*>(s_base + q1 * s_ld + c) = make_float2(s0[2] * scale_log2, s0[3] * scale_log2);
  };
  struct Sink2 { decltype(store)& f; __device__ __forceinline__ void operator()(int tile, const float (&s)[2][4]) const { f(tile, s[0], 0); f(tile, s[1], 1); } };
  struct Sink4 { decltype(store)& f; __device__ __forceinline__ void operator()(int tile, const float (&s)[4][4]) const { f(tile, s[0], 0); f(tile, s[1], 1); f(tile, s[2], 2); f(tile, s[3], 3); } };
  const Sink2 sink2{store};
  const Sink4 sink4{store};
  auto visible_in = [&](int tile) { return [=](int c, bool) { return tile * KT + c < n; }; };

  for (int it = 0; it < n_tiles; it += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (it + PRE + u < n_tiles) issue_tile(it + PRE + u);
      cp_async_commit();
    }
    cp_async_wait<PRE>();
    __syncwarp();
    const uint32_t ks = ring + (it % STAGES) * G::STAGE_B, vs = ks + G::TILE_B;
    const uint32_t ks2 = ring + ((it + 1) % STAGES) * G::STAGE_B, vs2 = ks2 + G::TILE_B;
    if ((it + 2) * KT <= n) {
      t.attend2(ks, vs, ks2, vs2, scale_log2, lane, sink4, it);
    } else {
      t.attend(ks, vs, scale_log2, lane, (it + 1) * KT > n, visible_in(it), sink2, it);
      if (it + 1 < n_tiles) t.attend(ks2, vs2, scale_log2, lane, true, visible_in(it + 1), sink2, it + 1);
    }
    __syncwarp();
  }
  cp_async_wait<0>();
  // ---- append: nothing in this launch reads the stored row
  if (newest >= 0 && newest < n && row0 == 0) {
    const int pt = newest / KT;
    const bool ok = __shfl_sync(0xffffffffu, (int)page_ok, pt) != 0;
    const int64_t dst = (((int64_t)__shfl_sync(0xffffffffu, page, pt) * KT + newest % KT) * a.Hkv + kvh) * D;
    if (ok && lane < 2 * CH) {
      const bf16* s = (lane < CH ? kn : vn) + ((int64_t)b * a.Hkv + kvh) * D;
      bf16* d = reinterpret_cast<bf16*>(lane < CH ? a.cache.k : a.cache.v) + dst;
      *reinterpret_cast<uint4*>(d + (lane % CH) * 8) = *reinterpret_cast<const uint4*>(s + (lane % CH) * 8);
    }
  }
  pdl_launch_dependents();
  t.reduce_sums();
  if constexpr (CLUSTER) {
    float* s_o = reinterpret_cast<float*>(smem);   // [16][D], over the ring
    float* s_ml = reinterpret_cast<float*>(smem + STAGES * G::STAGE_B + (WEIGH ? a.g * (a.chunk + 8) * 4 : 0));
    float *s_wt = s_ml + 32, *s_lse = s_wt + kMaxCluster * 16;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < NTILES; ++k) {
      *reinterpret_cast<float2*>(s_o + q0 * D + k * 8 + c2) = make_float2(t.o[k][0], t.o[k][1]);
      *reinterpret_cast<float2*>(s_o + q1 * D + k * 8 + c2) = make_float2(t.o[k][2], t.o[k][3]);
    }
    if ((lane & 3) == 0) {
      s_ml[q0] = t.m0; s_ml[q1] = t.m1;
      s_ml[16 + q0] = t.l0; s_ml[16 + q1] = t.l1;
    }
    cluster_arrive();
    cluster_wait();
    // lane r < g: row r's denominator over the whole list, and what each CTA's partial counts
    if (lane < a.g) {
      float m[kMaxCluster], mx = -INFINITY, sum = 0.f;
      const uint32_t at = ptx::smem_u32(s_ml + lane);
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) {
        m[k] = k < a.cluster ? peer_ld(peer_smem(at, k)) : -INFINITY;
        mx = fmaxf(mx, m[k]);
      }
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) {
        m[k] = ex2(m[k] - mx);
        if (k < a.cluster) sum += m[k] * peer_ld(peer_smem(at + 64, k));
      }
      const float inv = len > 0 ? 1.f / sum : 0.f;   // (a sequence without rows: zeros)
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) s_wt[k * 16 + lane] = m[k] * inv;
      s_lse[lane] = mx + log2f(sum);
    }
    __syncwarp();
    constexpr int V4 = D / 4;
    const uint32_t o_at = ptx::smem_u32(s_o);
    for (int i = split * 32 + lane; i < a.g * V4; i += a.cluster * 32) {
      const int r = i / V4;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) {
        if (k < a.cluster) {
          const float4 x = peer_ld4(peer_smem(o_at + i * 16, k));
          const float w = s_wt[k * 16 + r];
          acc.x = fmaf(w, x.x, acc.x); acc.y = fmaf(w, x.y, acc.y); acc.z = fmaf(w, x.z, acc.z); acc.w = fmaf(w, x.w, acc.w);
        }
      }
      reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(a.o) + ((int64_t)b * a.Hq + kvh * a.g) * D)[i] =
          make_uint2(pack2(acc.x, acc.y), pack2(acc.z, acc.w));
    }
    cluster_arrive();   // (what is left reads this CTA's own memory)
    const int64_t cap_row = ((int64_t)b * a.Hkv + kvh) * EARN_PAGE_TOKENS * a.cache.pages_per_seq;
    if (split == 0 && lane == 0 && a.pos != nullptr && len > 0) a.pos[cap_row + len - 1] = a.new_pos[b];
    if (WEIGH) {
      for (int j = lane * 4; j < n; j += 128) {
        float w[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < a.g; ++r) {
          const float4 x = *reinterpret_cast<const float4*>(s_base + r * s_ld + j);   // (columns past the list are not used)
          const float d = s_lse[r];
          w[0] += ex2(x.x - d); w[1] += ex2(x.y - d); w[2] += ex2(x.z - d); w[3] += ex2(x.w - d);
        }
        const float4 before = a.weight ? *reinterpret_cast<const float4*>(a.weight + cap_row + begin + j) : make_float4(0.f, 0.f, 0.f, 0.f);
        add_weights(a.weight_out + cap_row + begin + j, before, j, n, newest, w);
      }
    }
    cluster_wait();   // the other CTAs have read this one's shared memory
    return;
  }
  // ---- the partial: normalised rows and their log2-domain denominators
  const int64_t prow = (((int64_t)b * a.Hkv + kvh) * a.n_splits + split) * a.g;
  const float i0 = t.l0 == 0.f ? 0.f : 1.f / t.l0, i1 = t.l1 == 0.f ? 0.f : 1.f / t.l1;   // (0: every logit of the chunk is -inf)
  if (q0 < a.g) {
    float* p0 = a.part_o + (prow + q0) * D + c2;
#pragma unroll
    for (int k = 0; k < NTILES; ++k) *reinterpret_cast<float2*>(p0 + k * 8) = make_float2(t.o[k][0] * i0, t.o[k][1] * i0);
    if ((lane & 3) == 0) a.part_lse[prow + q0] = t.m0 + log2f(t.l0);
  }
  if (q1 < a.g) {
    float* p1 = a.part_o + (prow + q1) * D + c2;
#pragma unroll
    for (int k = 0; k < NTILES; ++k) *reinterpret_cast<float2*>(p1 + k * 8) = make_float2(t.o[k][2] * i1, t.o[k][3] * i1);
    if ((lane & 3) == 0) a.part_lse[prow + q1] = t.m1 + log2f(t.l1);
  }
}

// ------------------------------------------------------------------------------------------------ fp32
// 128 threads per (sequence, kv head, chunk, R query rows), tiles of 32 rows in shared memory, two in turn.  Logits: a lane per
// row of the tile, a warp per quarter of the columns, so that a K element is read once for all R query rows; the quarters
// are added through shared memory.  P V: a thread per column (at D = 64 each half of the CTA takes half the tile), a V element
// read once for all rows.  What bounds it is shared memory: 16 bytes of K per 4 R products.
constexpr int FT = 32;   // rows per tile
template <int D, int R>
struct F32Smem {
  static constexpr int PITCH = D + 4;   // floats; lanes a row apart hit different banks with 16-byte reads
  float k[2][FT][PITCH], v[2][FT][D];
  float q[R][D];
  float quarter[4][R][FT];
  float s[R][FT];
  float alpha[R], m[R], l[R];
};

template <int D, int R, bool WEIGH>
__global__ void __launch_bounds__(128) paged_decode_f32_kernel(PagedDecodeArgs a) {
  using S = F32Smem<D, R>;
  extern __shared__ __align__(128) uint8_t smem[];
  S& sh = *reinterpret_cast<S*>(smem);
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kvh = blockIdx.x, b = blockIdx.z;
  const int row_tiles = (a.g + R - 1) / R;
  const int split = blockIdx.y / row_tiles, row0 = (blockIdx.y % row_tiles) * R;
  const int rows = min(a.g - row0, R);
  const int len = paged_len(a.cache, b);
  const int begin = split * a.chunk, n = min(len - begin, a.chunk);
  if (n <= 0) return;
  const int n_tiles = (n + FT - 1) / FT;
  const float scale_log2 = a.scale * kLog2e;
  const float *kp = reinterpret_cast<const float*>(a.cache.k), *vp = reinterpret_cast<const float*>(a.cache.v);
  const float *kn = reinterpret_cast<const float*>(a.k_new), *vn = reinterpret_cast<const float*>(a.v_new);
  const int newest = kn != nullptr ? len - 1 - begin : -1;
  const int64_t new_off = ((int64_t)b * a.Hkv + kvh) * D;

  constexpr int CH = D / 4;   // 16-byte pieces of a row
  auto issue_tile = [&](int t) {
#pragma unroll
    for (int i = tid; i < FT * CH; i += 128) {
      const int r = i / CH, c = (i % CH) * 4, p = t * FT + r;
      bool ok;
      const int page = p < n ? paged_page(a.cache, b, (begin + p) / EARN_PAGE_TOKENS, ok) : 0;
      const int64_t off = (((int64_t)page * EARN_PAGE_TOKENS + p % EARN_PAGE_TOKENS) * a.Hkv + kvh) * D;   // (begin is a multiple of 16)
      const bool fresh = p == newest;
      cp_async16(ptx::smem_u32(&sh.k[t & 1][r][c]), (fresh ? kn + new_off : kp + off) + c, p < n ? 16 : 0);
      cp_async16(ptx::smem_u32(&sh.v[t & 1][r][c]), (fresh ? vn + new_off : vp + off) + c, p < n ? 16 : 0);
    }
    cp_async_commit();
  };
  issue_tile(0);
  for (int i = tid; i < R * D; i += 128)
    sh.q[i / D][i % D] = i / D < rows ? reinterpret_cast<const float*>(a.q)[((int64_t)b * a.Hq + kvh * a.g + row0) * D + i] : 0.f;
  constexpr int HALVES = 128 / D, JN = FT / HALVES;   // rows of the tile a thread takes in P V
  const int col = tid % D, half = tid / D;
  float acc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r] = 0.f;
  if (tid < R) { sh.m[tid] = -INFINITY; sh.l[tid] = 0.f; }
  float* s_base = WEIGH ? a.scores + ((int64_t)b * a.Hkv + kvh) * a.g * a.score_ld + begin : nullptr;

  for (int t = 0; t < n_tiles; ++t) {
    if (t + 1 < n_tiles) issue_tile(t + 1);
    else cp_async_commit();
    cp_async_wait<1>();
    __syncthreads();
    const int buf = t & 1, p = t * FT + lane;
    {
      float x[R];
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = 0.f;
      const int d0 = warp * (D / 4);
#pragma unroll
      for (int d = 0; d < D / 4; d += 4) {
        const float4 kk = *reinterpret_cast<const float4*>(&sh.k[buf][lane][d0 + d]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float4 qq = *reinterpret_cast<const float4*>(&sh.q[r][d0 + d]);
          x[r] = fmaf(kk.x, qq.x, x[r]); x[r] = fmaf(kk.y, qq.y, x[r]);
          x[r] = fmaf(kk.z, qq.z, x[r]); x[r] = fmaf(kk.w, qq.w, x[r]);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) sh.quarter[warp][r][lane] = x[r];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (R + 3) / 4; ++i) {   // softmax: a warp per query row
      const int r = warp + 4 * i;
      if (r < rows) {   // warp-uniform
        const float dot = (sh.quarter[0][r][lane] + sh.quarter[1][r][lane]) + (sh.quarter[2][r][lane] + sh.quarter[3][r][lane]);
        const float s = p < n ? dot * scale_log2 : -INFINITY;
        if (WEIGH && p < n) s_base[(int64_t)(row0 + r) * a.score_ld + p] = s;
        float mx = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float m = sh.m[r], mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn;
        const float al = exp2f(m - mu), e = exp2f(s - mu);
        float sum = e;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        sh.s[r][lane] = e;
        __syncwarp();
        if (lane == 0) { sh.alpha[r] = al; sh.m[r] = mn; sh.l[r] = sh.l[r] * al + sum; }
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] *= r < rows ? sh.alpha[r] : 0.f;
#pragma unroll 2
    for (int j = half * JN; j < (half + 1) * JN; j += 4) {
      const float v0 = sh.v[buf][j][col], v1 = sh.v[buf][j + 1][col], v2 = sh.v[buf][j + 2][col], v3 = sh.v[buf][j + 3][col];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r < rows) {
          const float4 pp = *reinterpret_cast<const float4*>(&sh.s[r][j]);
          acc[r] = fmaf(pp.x, v0, acc[r]); acc[r] = fmaf(pp.y, v1, acc[r]);
          acc[r] = fmaf(pp.z, v2, acc[r]); acc[r] = fmaf(pp.w, v3, acc[r]);
        }
      }
    }
    __syncthreads();   // the tile and the probabilities have been read
  }
  cp_async_wait<0>();
  if (newest >= 0 && newest < n && row0 == 0) {
    bool ok;
    const int page = paged_page(a.cache, b, (begin + newest) / EARN_PAGE_TOKENS, ok);
    const int64_t dst = (((int64_t)page * EARN_PAGE_TOKENS + newest % EARN_PAGE_TOKENS) * a.Hkv + kvh) * D;
    if (ok && tid < D) {
      reinterpret_cast<float*>(a.cache.k)[dst + tid] = kn[new_off + tid];
      reinterpret_cast<float*>(a.cache.v)[dst + tid] = vn[new_off + tid];
    }
  }
  pdl_launch_dependents();
  const int64_t prow = (((int64_t)b * a.Hkv + kvh) * a.n_splits + split) * a.g + row0;
  if (tid < rows) {
    sh.alpha[tid] = sh.l[tid] == 0.f ? 0.f : 1.f / sh.l[tid];   // (0: every logit of the chunk is -inf)
    a.part_lse[prow + tid] = sh.m[tid] + log2f(sh.l[tid]);
  }
  float* other = &sh.v[0][0][0];   // the second half's sums (D = 64)
  if (HALVES == 2 && half == 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) other[r * D + col] = acc[r];
  }
  __syncthreads();
  if (half == 0) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < rows) a.part_o[(prow + r) * D + col] = (HALVES == 2 ? acc[r] + other[r * D + col] : acc[r]) * sh.alpha[r];
  }
}

// ------------------------------------------------------------------------------------------------ join
// The first blocks of a (sequence, kv head) take ROWS output rows each, the warps shared out to them: the partials, weighted
// by 2^(their LSE - LSE of all).  The blocks behind them take KEYS rows of the list each: their weights.  Four rows and 2048
// keys a block, so that the blocks of a batch make one wave; one row and 1024 keys where the lists are few (and cut into many
// chunks: one list of 16384 rows, 8 kv heads: 30 us with the wide blocks).  What a block
// reads does not depend on the length (only what it uses does), so the denominators, partials and logits are all asked for
// at once: one round trip to L2 instead of the chain length -> denominators -> partials, and few enough blocks for one wave.
constexpr int JOIN_THREADS = 256, JOIN_AHEAD = 4, JOIN_MAX_G = 1024;
template <bool FEW>
struct Join {
  static constexpr int ROWS = FEW ? 1 : 4, KEYS = (FEW ? 4 : 8) * JOIN_THREADS;
};

// log2-domain denominator of query row r over `live` splits, by one warp; x0, x1: the lane's splits lane and lane + 32
__device__ __forceinline__ float join_lse(const float* lse, int g, int r, int live, int lane, float x0, float x1) {
  x0 = lane < live ? x0 : -INFINITY;
  x1 = lane + 32 < live ? x1 : -INFINITY;
  float mx = fmaxf(x0, x1);
  for (int s = lane + 64; s < live; s += 32) mx = fmaxf(mx, lse[s * g + r]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  const float mu = mx == -INFINITY ? 0.f : mx;
  float sum = ex2(x0 - mu) + ex2(x1 - mu);
  for (int s = lane + 64; s < live; s += 32) sum += ex2(lse[s * g + r] - mu);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return mu + log2f(sum);
}

template <typename T, int D, bool FEW>
__global__ void __launch_bounds__(JOIN_THREADS) paged_join_kernel(PagedDecodeArgs a) {
  constexpr int JOIN_ROWS = Join<FEW>::ROWS, JOIN_KEYS = Join<FEW>::KEYS, HALVES = JOIN_KEYS / (4 * JOIN_THREADS), WPR = JOIN_THREADS / 32 / JOIN_ROWS;
  __shared__ float lse_all[JOIN_MAX_G];
  __shared__ float4 part[JOIN_THREADS];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kvh = blockIdx.y, b = blockIdx.z, g = a.g;
  const int64_t unit = (int64_t)b * a.Hkv + kvh;
  const float* lse = a.part_lse + unit * a.n_splits * g;
  const int o_blocks = (g + JOIN_ROWS - 1) / JOIN_ROWS;
  if ((int)blockIdx.x < o_blocks) {
    constexpr int V4 = D / 4, SUB = 32 / V4, STEP = WPR * SUB, AHEAD = 4;   // float4 per row; splits a warp, a row's warps take at once
    const int r = (int)blockIdx.x * JOIN_ROWS + warp / WPR;
    const int first = warp % WPR * SUB + lane / V4;
    const float4* po = reinterpret_cast<const float4*>(a.part_o) + (unit * a.n_splits * g + r) * V4 + lane % V4;
    const bool in = r < g;
    float4 y[AHEAD];
    float ly[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int s = first + k * STEP;
      const bool ok = in && s < a.n_splits;
      ly[k] = ok ? lse[s * g + r] : 0.f;
      y[k] = ok ? po[(int64_t)s * g * V4] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const float x0 = in && lane < a.n_splits ? lse[lane * g + r] : 0.f, x1 = in && lane + 32 < a.n_splits ? lse[(lane + 32) * g + r] : 0.f;
    const int len = paged_len(a.cache, b), live = (len + a.chunk - 1) / a.chunk;   // splits that hold rows
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in) {   // (warp-uniform)
      const float all = join_lse(lse, g, r, live, lane, x0, x1);
      auto add = [&](float l, const float4& z) {
        const float w = ex2(l - all);
        acc.x = fmaf(w, z.x, acc.x); acc.y = fmaf(w, z.y, acc.y); acc.z = fmaf(w, z.z, acc.z); acc.w = fmaf(w, z.w, acc.w);
      };
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (first + k * STEP < live) add(ly[k], y[k]);
#pragma unroll 8
      for (int s = first + AHEAD * STEP; s < live; s += STEP) add(lse[s * g + r], po[(int64_t)s * g * V4]);
    }
    part[tid] = acc;
    __syncthreads();
    if (in && warp % WPR == 0 && lane < V4) {
      float o[4] = {0.f, 0.f, 0.f, 0.f};   // (a sequence without rows: zeros)
#pragma unroll
      for (int k = 0; k < STEP; ++k) {
        const float4 z = part[warp * 32 + k * V4 + lane];
        o[0] += z.x; o[1] += z.y; o[2] += z.z; o[3] += z.w;
      }
      Elem<T>::store4(reinterpret_cast<T*>(a.o) + ((int64_t)b * a.Hq + kvh * g + r) * D + lane * 4, o);
    }
    if (blockIdx.x == 0 && tid == 0 && a.pos != nullptr && len > 0)
      a.pos[unit * EARN_PAGE_TOKENS * a.cache.pages_per_seq + len - 1] = a.new_pos[b];
    return;
  }
  // ---- weights
  const int key0 = ((int)blockIdx.x - o_blocks) * JOIN_KEYS + tid * 4;
  const float* sc = a.scores + unit * g * a.score_ld + key0;
  float4 x[HALVES][JOIN_AHEAD];
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int r = 0; r < JOIN_AHEAD; ++r)
      if (r < g && key0 + h * (4 * JOIN_THREADS) < a.score_ld)
        x[h][r] = *reinterpret_cast<const float4*>(sc + (int64_t)r * a.score_ld + h * (4 * JOIN_THREADS));   // (columns past the list are not used)
  const int64_t row0 = unit * EARN_PAGE_TOKENS * a.cache.pages_per_seq;
  float4 in[HALVES];
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    in[h] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.weight && key0 + h * (4 * JOIN_THREADS) < a.score_ld) in[h] = *reinterpret_cast<const float4*>(a.weight + row0 + key0 + h * (4 * JOIN_THREADS));
  }
  const int len = paged_len(a.cache, b), live = (len + a.chunk - 1) / a.chunk;
  for (int r = warp; r < g; r += JOIN_THREADS / 32) {
    const float x0 = lane < a.n_splits ? lse[lane * g + r] : 0.f, x1 = lane + 32 < a.n_splits ? lse[(lane + 32) * g + r] : 0.f;
    const float all = join_lse(lse, g, r, live, lane, x0, x1);
    if (lane == 0) lse_all[r] = all;
  }
  __syncthreads();
  const int fresh = a.k_new != nullptr ? len - 1 : -1;   // the appended row starts from zero
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    const int j = key0 + h * (4 * JOIN_THREADS);
    if (j >= len) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float4& y, float d) { w[0] += ex2(y.x - d); w[1] += ex2(y.y - d); w[2] += ex2(y.z - d); w[3] += ex2(y.w - d); };
#pragma unroll
    for (int r = 0; r < JOIN_AHEAD; ++r)
      if (r < g) add(x[h][r], lse_all[r]);
#pragma unroll 4
    for (int r = JOIN_AHEAD; r < g; ++r)
      add(*reinterpret_cast<const float4*>(sc + (int64_t)r * a.score_ld + h * (4 * JOIN_THREADS)), lse_all[r]);
    add_weights(a.weight_out + row0 + j, in[h], j, len, fresh, w);
  }
}

// cluster form: a.cluster CTAs per (sequence, kv head), launched as one cluster
template <int D, bool WEIGH>
cudaError_t launch_cluster(const PagedDecodeArgs& a, cudaStream_t st) {
  const int smem = cluster_smem<D>(a.g, a.chunk, WEIGH);
  cudaError_t e = ensure_dynamic_smem<paged_decode_kernel<D, WEIGH, true>>(cluster_smem<D>(16, kPagedMaxChunk, WEIGH));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(a.Hkv * a.cluster, 1, a.n_seq);
  cfg.blockDim = dim3(32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, paged_decode_kernel<D, WEIGH, true>, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D, bool WEIGH>
cudaError_t launch_main(const PagedDecodeArgs& a, cudaStream_t st) {
  const dim3 grid(a.Hkv, a.n_splits * ((a.g + 15) / 16), a.n_seq);
  cudaError_t e;
  if (a.dtype == EARN_BF16) {
    constexpr int smem = STAGES * Geo<D>::STAGE_B;
    e = ensure_dynamic_smem<paged_decode_kernel<D, WEIGH, false>>(smem);
    if (e == cudaSuccess) e = launch_pdl(paged_decode_kernel<D, WEIGH, false>, grid, dim3(32), smem, st, a);
  } else {
    // query rows per CTA: four if the group has no more (fewer idle products), else sixteen
    auto launch = [&](auto rows_tag) {
      constexpr int R = decltype(rows_tag)::value;
      constexpr int smem = (int)sizeof(F32Smem<D, R>);
      cudaError_t err = ensure_dynamic_smem<paged_decode_f32_kernel<D, R, WEIGH>>(smem);
      if (err == cudaSuccess)
        err = launch_pdl(paged_decode_f32_kernel<D, R, WEIGH>, dim3(a.Hkv, a.n_splits * ((a.g + R - 1) / R), a.n_seq), dim3(128), smem, st, a);
      return err;
    };
    e = a.g <= 4 ? launch(std::integral_constant<int, 4>{}) : launch(std::integral_constant<int, 16>{});
  }
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const PagedDecodeArgs& a, cudaStream_t st) {
  if (a.cluster > 0) return a.weight_out ? launch_cluster<D, true>(a, st) : launch_cluster<D, false>(a, st);
  cudaError_t e = a.weight_out ? launch_main<D, true>(a, st) : launch_main<D, false>(a, st);
  if (e != cudaSuccess) return e;
  auto join = [&](auto few_tag) {
    constexpr bool FEW = decltype(few_tag)::value;
    constexpr int ROWS = Join<FEW>::ROWS, KEYS = Join<FEW>::KEYS;
    const dim3 grid((a.g + ROWS - 1) / ROWS + (a.weight_out ? (a.cache.max_len + KEYS - 1) / KEYS : 0), a.Hkv, a.n_seq);
    return a.dtype == EARN_BF16 ? launch_pdl(paged_join_kernel<bf16, D, FEW>, grid, dim3(JOIN_THREADS), 0, st, a)
                                : launch_pdl(paged_join_kernel<float, D, FEW>, grid, dim3(JOIN_THREADS), 0, st, a);
  };
  e = (int64_t)a.n_seq * a.Hkv * a.g <= 2 * sm_count() ? join(std::true_type{}) : join(std::false_type{});
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// A call with less work than a wave of chunks is a chain of latencies, and one launch with the join inside the cluster beats
// two: 64 (sequence, kv head) pairs of 1000 rows 12.0 us against 14.7, 192 of 50 to 200 rows 8.7 against 9.4 (group of 7),
// 512 of 300 rows 22.4 against 23.7.  Past that a cluster's CTAs sit out the exchange without a load in flight (512 pairs of
// 700 to 1044 rows: 54.5 us against 51.3), and more than 256 rows a warp take too long (16 pairs of 2000 rows: level).
PagedPlan plan_paged_decode(int n_seq, int n_kv_heads, int g, int max_len, int dtype) {
  PagedPlan p{};
  const int64_t units = (int64_t)n_seq * n_kv_heads * ((g + 15) / 16), sms = sm_count();
  constexpr int ROWS = kPagedMaxChunk / 2;
  if (dtype == EARN_BF16 && g <= 16 && max_len <= kMaxCluster * ROWS && units * max_len <= 6 * sms * ROWS) {
    int c = 1;   // enough CTAs for half the warp slots, unless their lists come to less than two tiles
    while (c < kMaxCluster && ((max_len + c - 1) / c > ROWS || (units * c < 3 * sms && max_len > 2 * KT * c))) c *= 2;
    p.cluster = c;
    p.chunk = ((max_len + KT - 1) / KT + c - 1) / c * KT;
    return p;
  }
  // One chunk per warp slot (six one-warp CTAs an SM) while that leaves it at most 256 rows; otherwise about three chunks per
  // slot, so that uneven lists even out, of 160 to 512 rows.
  int64_t c = (units * max_len + 6 * sms - 1) / (6 * sms);
  if (c > kPagedMaxChunk / 2) c = c / 3 < 160 ? 160 : c / 3;
  c = (c + 31) / 32 * 32;
  c = c < 32 ? 32 : c > kPagedMaxChunk ? kPagedMaxChunk : c;
  p.chunk = (int)c;
  p.n_splits = (int)((max_len + c - 1) / c);
  return p;
}

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, cudaStream_t st) {
  return a.D == 64 ? launch_d<64>(a, st) : launch_d<128>(a, st);
}

}  // namespace earn

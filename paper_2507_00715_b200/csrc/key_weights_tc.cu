// Accumulated attention weight of the prompt's rows (earn_key_weights) on the Blackwell tensor cores: bf16 Q and K,
// head_dim 64 or 128, fp32 logits, exponentials and sums.
//
//   weight[h, j] = sum over the window's queries i >= j and the heads a of h's group of exp(q_ia . k_jh * scale - lse_ai)
//
// The logits are computed transposed, S^T = K Q^T, keys along the 128 rows of the accumulator: a softmax thread then owns
// one key and sums along its own TMEM lane, with no exchange between threads until one 4-byte store per key.  The columns
// are (token, head of the group) pairs -- g heads of a token are contiguous in Q, so one TMA box of T = 128 / g tokens is a
// tile of T g columns, and a window of a few queries fills one tile for the whole group.
//
// Work item = 256 keys of one (sequence, kv head) (two accumulators that share every Q tile), over all Q tiles of the window
// that see them.  A planning kernel lists the blocks, most queries first; the main kernel is persistent, one CTA per SM.
//   warp 0      TMA: the two K tiles of the next item (double-buffered), a ring of Q tiles
//   warp 2      the softmax denominators of a Q tile's columns, negated and scaled into the log2 domain -> shared memory
//   warp 1      one thread issues tcgen05.mma into two TMEM buffers per accumulator
//   warps 4..   two warpgroups per accumulator, 64 columns each: 2^(S * scale - lse) summed per key
// Bound by the special-function unit and the tensor core (a tile of 128 x 128 logits costs 1024 clocks of exponentials at
// 16 per clock against 512 of MMA at D = 128) when the window is long; when it is short by neither HBM (0.77 of a copy) nor
// that unit (58 % busy) but by the two in turns, item by item.  Times in this file are of calls replayed from a graph: 8 x 4096
// tokens 621 us, 727 issued one by one for a while, when the power cap sets the clock.
//
// Every mbarrier wait is bounded; when one runs out the CTA raises its abort flag, writes EARN_ERR_TIMEOUT to the status
// word, drains what it has in flight, frees its TMEM and returns.
#include <algorithm>
#include <type_traits>

#include "paged_cache.cuh"
#include "sm100_ptx.cuh"
#include "tc_maps.cuh"

namespace earn {
namespace {
using namespace ptx;

constexpr int BM = 128, BC = 128, NT = 2;          // keys per accumulator, columns per Q tile, accumulators per item
constexpr float kLog2eRest = (float)(1.4426950408889634 - (double)kLog2e);   // (1.3e-8 of a denominator of 16 is 2e-7 of a weight)
constexpr long long WAIT_LIMIT = 2000000000LL;     // about one second of SM clocks

template <int HD>
struct Cfg {
  static constexpr int HALF = BM * 128;              // one 64-column block of a tile (128 rows x 128 B)
  static constexpr int TILE = HALF * (HD / 64);
  static constexpr int NSTAGE = 3;                   // Q ring
  static constexpr int OFF_K = 0;                    // [2][NT] tiles
  static constexpr int OFF_Q = OFF_K + 2 * NT * TILE;
  static constexpr int OFF_LSE = OFF_Q + NSTAGE * TILE;
  static constexpr int OFF_SUM = OFF_LSE + NSTAGE * BC * 4;   // [NT][128] halves of the keys' sums
  static constexpr int OFF_BAR = OFF_SUM + NT * BM * 4;
  static constexpr int SMEM_BYTES = OFF_BAR + 256;
  static constexpr int TMEM_COLS = NT * 2 * BC;
  static constexpr int THREADS = 32 * (4 + 8 * NT);
  static constexpr int BAR_KFULL = 0, BAR_KFREE = 2, BAR_QFULL = 4, BAR_QFREE = BAR_QFULL + NSTAGE, BAR_LFULL = BAR_QFREE + NSTAGE,
                       BAR_LFREE = BAR_LFULL + NSTAGE, BAR_SFULL = BAR_LFREE + NSTAGE, BAR_SFREE = BAR_SFULL + 2 * NT,
                       BAR_SUM = BAR_SFREE + 2 * NT, BAR_SUMFREE = BAR_SUM + NT, BAR_DRAIN = BAR_SUMFREE + NT, N_BARS = BAR_DRAIN + 1;
  static_assert(8 * N_BARS + 16 <= 256 && SMEM_BYTES <= 232448, "shared memory");
};

// Where the blocks of each sequence start in the list of all blocks, for short windows (every block has about the same work, so
// they need no sorting) of batches that fit a kernel parameter: no planning kernel, one launch (6.6 -> 4.9 us for one prompt,
// 71 -> 67 us for 32-row windows of 128 ragged ones).
constexpr int TABLE_SEQS = 256;
struct KwTable {
  int first[TABLE_SEQS + 1];
};

struct KwParams {
  const float* lse;
  float* weight;
  const int4* plan;          // {first global row of the block, rows of the sequence from there, block, sequence}, or null: the table
  const int32_t* cu_seqlens;
  int32_t* status;
  int batch, Hq, Hkv, g, T, n_obs, total, n_items;
  float scale_log2;
};

struct Item {
  int lo, len, kvh;   // the sequence's first row and length
  int key0;           // first key of the block (position in the sequence)
  int first;          // first query of the window that sees any of these keys
  int n_qt;           // Q tiles
};

// The planner orders blocks by their number, highest first (for queries that is the longest key range).  Here block t has
// the more queries the lower it is, so the order is read backwards within the sequence.
__device__ __forceinline__ Item load_item(const KwParams& p, const KwTable& table, int i) {
  const int e = i / p.Hkv;
  Item it;
  it.kvh = i - e * p.Hkv;
  if (p.plan != nullptr) {
    const int4 t = __ldg(p.plan + e);
    it.lo = __ldg(p.cu_seqlens + t.w);
    it.len = t.z * (NT * BM) + t.y;
    it.key0 = ((it.len + NT * BM - 1) / (NT * BM) - 1 - t.z) * (NT * BM);
  } else {
    int b = 0;   // the last sequence whose blocks start at or before e (one without blocks starts where the next one does)
    for (int step = TABLE_SEQS / 2; step > 0; step >>= 1)
      if (b + step < p.batch && table.first[b + step] <= e) b += step;
    it.lo = __ldg(p.cu_seqlens + b);
    it.len = __ldg(p.cu_seqlens + b + 1) - it.lo;
    it.key0 = (e - table.first[b]) * (NT * BM);
  }
  it.first = max(max(it.len - p.n_obs, 0), it.key0);
  it.n_qt = (it.len - it.first + p.T - 1) / p.T;
  return it;
}
// Does accumulator x take part in Q tile i: does the tile's last query see the accumulator's first key?
__device__ __forceinline__ bool active(const KwParams& p, const Item& it, int x, int i) {
  return min(it.first + (i + 1) * p.T, it.len) - 1 >= it.key0 + x * BM;
}

// (d0, d1) = (a0, a1) * b + (c0, c1), (d0, d1) += (a0, a1): packed fp32 pairs
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c0, float c1) {
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %6};\n\t"
      "fma.rn.ftz.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void add2(float& d0, float& d1, float a0, float a1) {
  asm("{\n\t.reg .b64 ra, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rd, {%0, %1};\n\tadd.rn.ftz.f32x2 rd, rd, ra;\n\t"
      "mov.b64 {%0, %1}, rd;\n\t}"
      : "+f"(d0), "+f"(d1) : "f"(a0), "f"(a1));
}

template <int HD>
__global__ void __launch_bounds__(Cfg<HD>::THREADS, 1)
key_weights_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_pad,
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ KwTable table, KwParams p) {
  using C = Cfg<HD>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];   // (swizzled tiles need 1024-byte alignment)
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* gen = smem_raw;
  const uint32_t sK = base + C::OFF_K, sQ = base + C::OFF_Q, bars = base + C::OFF_BAR;
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + C::OFF_BAR + 8 * C::N_BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + C::OFF_BAR + 8 * C::N_BARS + 8);
  float* s_lse = reinterpret_cast<float*>(gen + C::OFF_LSE);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile_rows = p.T * p.g;                        // columns that belong to a token
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(C::BAR_KFULL + s), 1);
      mbar_init(bar(C::BAR_KFREE + s), 1);
    }
    for (int s = 0; s < C::NSTAGE; ++s) {
      mbar_init(bar(C::BAR_QFULL + s), 1);
      mbar_init(bar(C::BAR_QFREE + s), 1);
      mbar_init(bar(C::BAR_LFULL + s), 32);
      mbar_init(bar(C::BAR_LFREE + s), 8 * NT);
    }
    for (int s = 0; s < 2 * NT; ++s) {
      mbar_init(bar(C::BAR_SFULL + s), 1);
      mbar_init(bar(C::BAR_SFREE + s), 8);
    }
    for (int x = 0; x < NT; ++x) {
      mbar_init(bar(C::BAR_SUM + x), 4);
      mbar_init(bar(C::BAR_SUMFREE + x), 4);
    }
    mbar_init(bar(C::BAR_DRAIN), 1);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int n_cta = gridDim.x;
  // passes of gridDim.x items, forwards and backwards in turn: the list is sorted, most work first
  auto item_at = [&](int k) { return k * n_cta + ((k & 1) ? n_cta - 1 - (int)blockIdx.x : (int)blockIdx.x); };
  pdl_launch_dependents();
  pdl_wait();   // the plan (written by the kernel launched just before this one) and every tensor are read below
  // Item k of this CTA, for a whole warp: the lanes look 32 items up side by side and hand them out by shuffle.  (A look-up
  // is a chain of reads of 1000 clocks and more, and a warp stalls on it where it stands: with one an item, 70 us for the
  // 32-row windows of 128 ragged prompts.)
  Item mine{};
  int mine_from = INT32_MIN / 2;
  auto look_up = [&](int k) {
    if (k - mine_from >= 32) {
      mine_from = k;
      mine = load_item(p, table, min(item_at(k + lane), p.n_items - 1));
    }
    const int from = k - mine_from;
    Item it;
    it.lo = __shfl_sync(0xffffffffu, mine.lo, from);
    it.len = __shfl_sync(0xffffffffu, mine.len, from);
    it.kvh = __shfl_sync(0xffffffffu, mine.kvh, from);
    it.key0 = __shfl_sync(0xffffffffu, mine.key0, from);
    it.first = __shfl_sync(0xffffffffu, mine.first, from);
    it.n_qt = __shfl_sync(0xffffffffu, mine.n_qt, from);
    return it;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (lane 0 issues)
    const bool leader = lane == 0;
    auto wait = [&](int b, int parity) {   // warp-uniform result
      return __all_sync(0xffffffffu, mbar_wait_bounded(bar(b), (uint32_t)parity & 1u, abort_flag, WAIT_LIMIT));
    };
    int e = 0, n = 0;   // Q tiles and items issued so far
    bool ok = true;
    while (item_at(n) < p.n_items && ok) {
      const Item it = look_up(n);
      const int kb = n & 1;
      if (n >= 2) ok = wait(C::BAR_KFREE + kb, (n >> 1) - 1);
      if (!ok) break;
      if (leader) {
        const int tiles = it.key0 + BM < it.len ? NT : 1;   // the second accumulator may lie past the sequence
        mbar_expect_tx(bar(C::BAR_KFULL + kb), tiles * C::TILE);
        for (int x = 0; x < tiles; ++x)
          for (int h = 0; h < HD / 64; ++h)
            tma_load_3d(sK + (kb * NT + x) * C::TILE + h * C::HALF, &map_k, bar(C::BAR_KFULL + kb), h * 64, it.kvh, it.lo + it.key0 + x * BM);
      }
      ++n;
      for (int t = 0; t < it.n_qt; ++t, ++e) {
        const int st = e % C::NSTAGE;
        if (e >= C::NSTAGE) ok = wait(C::BAR_QFREE + st, (e / C::NSTAGE) - 1);
        if (!ok) break;
        if (leader) {
          mbar_expect_tx(bar(C::BAR_QFULL + st), C::TILE);
          for (int h = 0; h < HD / 64; ++h)
            tma_load_3d(sQ + st * C::TILE + h * C::HALF, &map_q, bar(C::BAR_QFULL + st), h * 64, it.kvh * p.g, it.lo + it.first + t * p.T);
          // The columns left over (128 is not a multiple of g) take rows of the tile's last token once more, against a
          // denominator of +inf.  Any key that sees them sees that token, so they add a 0 unless it adds a NaN or an
          // infinity itself; a row of zeros would turn an infinite key, whose weight may be 0, into a NaN.
          if (tile_rows < BC) {
            const int last = it.lo + min(it.first + (t + 1) * p.T, it.len) - 1;
            for (int h = 0; h < HD / 64; ++h)
              tma_load_3d(sQ + st * C::TILE + h * C::HALF + tile_rows * 128, &map_pad, bar(C::BAR_QFULL + st), h * 64, it.kvh * p.g, last);
          }
        }
      }
    }
    if (leader && *abort_flag) {
      // let the copies already in flight land before the CTA gives its shared memory back
      int none = 0;
      for (int f = max(e - C::NSTAGE, 0); f < e; ++f) mbar_wait_bounded(bar(C::BAR_QFULL + f % C::NSTAGE), (f / C::NSTAGE) & 1, &none, WAIT_LIMIT);
      for (int f = max(n - 2, 0); f < n; ++f) mbar_wait_bounded(bar(C::BAR_KFULL + (f & 1)), (f >> 1) & 1, &none, WAIT_LIMIT);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------------ denominators of the columns
    int tok[4];
    int64_t at[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int col = lane + 32 * c;
      tok[c] = col < tile_rows ? col / p.g : INT32_MAX / 2;
      at[c] = (int64_t)(col % p.g) * p.total + (col < tile_rows ? col / p.g : 0);
    }
    auto fetch = [&](float (&v)[4], const Item& it, int t) {
      const float* src = p.lse + (int64_t)it.kvh * p.g * p.total + it.lo;
      const int tok0 = it.first + t * p.T;
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = tok0 + tok[c] < it.len ? __ldg(src + at[c] + tok0) : INFINITY;
    };
    int e = 0;
    bool ok = true;
    Item it = look_up(0);
    float cur[4], nxt[4];
    if (item_at(0) < p.n_items) fetch(cur, it, 0);
    for (int n = 0; item_at(n) < p.n_items && ok; ++n) {
      const Item nxt_it = look_up(n + 1);
      for (int t = 0; t < it.n_qt; ++t, ++e) {
        // the next tile's denominators, of this item or the next, are in flight while this tile's slot comes free
        if (t + 1 < it.n_qt) fetch(nxt, it, t + 1);
        else if (item_at(n + 1) < p.n_items) fetch(nxt, nxt_it, 0);
        const int st = e % C::NSTAGE;
        if (e >= C::NSTAGE &&
            !__all_sync(0xffffffffu, mbar_wait_bounded(bar(C::BAR_LFREE + st), ((e / C::NSTAGE) - 1) & 1, abort_flag, WAIT_LIMIT))) {
          ok = false;
          break;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) s_lse[st * BC + lane + 32 * c] = fmaf(cur[c], -kLog2e, cur[c] * -kLog2eRest);
        mbar_arrive(bar(C::BAR_LFULL + st));
#pragma unroll
        for (int c = 0; c < 4; ++c) cur[c] = nxt[c];
      }
      it = nxt_it;
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    const bool leader = lane == 0;
    constexpr uint32_t idesc = idesc_bf16_f32(BM, BC, 0, 0);   // K (K-major) x Q^T (K-major); all columns, also those that no token fills
    constexpr uint32_t desc_hi = smem_desc_hi_sw128(1024);
    const uint32_t k_lo = smem_desc_lo(sK, 16), q_lo = smem_desc_lo(sQ, 16);
    auto wait = [&](int b, int parity) {   // warp-uniform result
      return __all_sync(0xffffffffu, mbar_wait_bounded(bar(b), (uint32_t)parity & 1u, abort_flag, WAIT_LIMIT));
    };
    int e = 0, ns[NT] = {0, 0};
    bool ok = true;
    for (int n = 0; item_at(n) < p.n_items && ok; ++n) {
      const Item it = look_up(n);
      const int kb = n & 1;
      ok = wait(C::BAR_KFULL + kb, n >> 1);
      for (int t = 0; t < it.n_qt && ok; ++t, ++e) {
        const int st = e % C::NSTAGE;
        ok = wait(C::BAR_QFULL + st, e / C::NSTAGE);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          if (!ok || !active(p, it, x, t)) continue;
          const int buf = ns[x] & 1;
          if (ns[x] >= 2) ok = wait(C::BAR_SFREE + x * 2 + buf, (ns[x] >> 1) - 1);
          if (!ok) continue;
          ++ns[x];
          tc_fence_after();
          const uint32_t a0 = k_lo + (kb * NT + x) * (C::TILE >> 4), b0 = q_lo + st * (C::TILE >> 4);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint32_t off = ((kk >> 2) * C::HALF + (kk & 3) * 32) >> 4;
              umma_ss_lohi(tmem + (x * 2 + buf) * BC, a0 + off, desc_hi, b0 + off, desc_hi, idesc, kk > 0);
            }
            umma_commit(bar(C::BAR_SFULL + x * 2 + buf));
          }
        }
        if (leader && ok) umma_commit(bar(C::BAR_QFREE + st));
      }
      if (leader && ok) umma_commit(bar(C::BAR_KFREE + kb));
    }
    if (leader && *abort_flag) {
      int none = 0;
      umma_commit(bar(C::BAR_DRAIN));   // everything this thread issued has retired once this fires
      mbar_wait_bounded(bar(C::BAR_DRAIN), 0, &none, WAIT_LIMIT);
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ one key per thread, half of a tile's columns
    const int x = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1;
    const int wq = warp & 3;            // a warp may only touch TMEM lanes 32*(warp % 4) ..
    const uint32_t t_s = tmem + ((uint32_t)(wq * 32) << 16) + x * 2 * BC + half * 64;
    float* s_sum = reinterpret_cast<float*>(gen + C::OFF_SUM) + x * BM + wq * 32 + lane;
    const float sl2 = p.scale_log2;
    int tok_lo[2], tok_hi[2];   // first and last token of the half's two 32-column chunks
#pragma unroll
    for (int q = 0; q < 2; ++q) { tok_lo[q] = (half * 64 + q * 32) / p.g; tok_hi[q] = (half * 64 + q * 32 + 31) / p.g; }
    int e = 0, ns = 0;
    bool ok = true;
    for (int n = 0; item_at(n) < p.n_items && ok; ++n) {
      const Item it = look_up(n);
      const int key = it.key0 + x * BM + wq * 32 + lane, key_hi = it.key0 + x * BM + wq * 32 + 31;   // this thread's, the warp's last
      float acc0 = 0.f, acc1 = 0.f;
      for (int t = 0; t < it.n_qt; ++t, ++e) {
        const int st = e % C::NSTAGE;
        // (a warp that skips the tile waits for its denominators all the same: it must not arrive twice in one phase)
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar(C::BAR_LFULL + st), (e / C::NSTAGE) & 1, abort_flag, WAIT_LIMIT));
        if (!ok) break;
        if (!active(p, it, x, t)) {   // warp-uniform
          if (lane == 0) mbar_arrive(bar(C::BAR_LFREE + st));
          continue;
        }
        const int buf = ns & 1;
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar(C::BAR_SFULL + x * 2 + buf), (ns >> 1) & 1, abort_flag, WAIT_LIMIT));
        if (!ok) break;
        ++ns;
        tc_fence_after();
        const int tok0 = it.first + t * p.T, toks = min(p.T, it.len - tok0);
        // columns [c_lo, c_lo + width) of this half are visible to this key: tokens at or after it, tokens of the sequence
        const int c_lo = max(key - tok0, 0) * p.g - half * 64;
        const uint32_t width = (uint32_t)max(toks * p.g - half * 64 - c_lo, 0);
        // A tile's terms are summed by themselves first: a chain over all of a long window's terms rounds each of them at the
        // size of the whole sum (4096 tokens, groups of 4: 1.0e-6 off, and 5.6e-7 this way; 8192, groups of 8: 1.7e-6, 5.4e-7).
        float sum0 = 0.f, sum1 = 0.f;
        const float4* l4 = reinterpret_cast<const float4*>(s_lse + st * BC + half * 64);
        uint32_t a[32];
        auto load = [&](int q) {
          tmem_ld_32x32(t_s + buf * BC + q * 32, a);
          tmem_wait_ld(a);
        };
        auto release = [&]() {   // the accumulator is free as soon as it has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::BAR_SFREE + x * 2 + buf));
        };
        auto add_all = [&](int q) {
#pragma unroll
          for (int c = 0; c < 32; c += 4) {
            const float4 l = l4[q * 8 + (c >> 2)];
            float e0, e1, e2, e3;
            // (subtracting in the natural domain and multiplying by log2 e afterwards: 3 % slower)
            fma2(e0, e1, __uint_as_float(a[c]), __uint_as_float(a[c + 1]), sl2, l.x, l.y);
            fma2(e2, e3, __uint_as_float(a[c + 2]), __uint_as_float(a[c + 3]), sl2, l.z, l.w);
            add2(sum0, sum1, ex2(e0), ex2(e1));   // (a share of the exponentials as polynomials on the FMA pipe: no faster,
            add2(sum0, sum1, ex2(e2), ex2(e3));   // 620 us with none, 643 with a quarter, 729 with half at 8 x 4096 tokens)
          }
        };
        // The interior takes straight-line code of its own: with a test per chunk in between, 641 us instead of 620.
        if (toks == p.T && tok0 >= key_hi) {
          load(0);
          add_all(0);
          load(1);
          release();
          add_all(1);
        } else {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            // (warp-uniform) a chunk none of whose tokens any of the warp's keys sees, or all of them, or some
            if (tok_lo[q] >= toks || tok0 + tok_hi[q] < key_hi - 31) continue;
            load(q);
            if (tok0 + tok_lo[q] >= key_hi && (toks == p.T || tok_hi[q] < toks)) {
              add_all(q);
              continue;
            }
            // what is not visible may be anything, a NaN included: it is selected away
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              const float4 l = l4[q * 8 + (c >> 2)];
              const float ll[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float v = ex2(fmaf(__uint_as_float(a[c + k]), sl2, ll[k]));
                sum0 += (uint32_t)(q * 32 + c + k - c_lo) < width ? v : 0.f;
              }
            }
          }
          release();
        }
        add2(acc0, acc1, sum0, sum1);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::BAR_LFREE + st));
      }
      if (!ok) break;
      // ---- the two halves of a key's sum meet in shared memory
      if (half == 1) {
        if (n > 0) ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar(C::BAR_SUMFREE + x), (n - 1) & 1, abort_flag, WAIT_LIMIT));
        if (!ok) break;
        *s_sum = acc0 + acc1;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::BAR_SUM + x));
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar(C::BAR_SUM + x), n & 1, abort_flag, WAIT_LIMIT));
        if (!ok) break;
        const float other = *s_sum;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::BAR_SUMFREE + x));
        if (key < it.len) p.weight[(int64_t)it.kvh * p.total + it.lo + key] = (acc0 + acc1) + other;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.status, (int32_t)EARN_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// packed [total, heads, HD] bf16 as tcmap::make_map describes it, but with boxes of `box_heads` heads
inline bool make_map(CUtensorMap* map, const void* ptr, int heads, int total, int head_dim, int box_heads, int box_rows) {
  auto fn = tcmap::encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)total};
  cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)heads * head_dim * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
cudaError_t launch_hd(const KeyWeightArgs& a, int plan_entries, void* plan, int32_t* status, cudaStream_t st) {
  const int g = a.Hq / a.Hkv, T = BC / g;
  CUtensorMap mq, mk;
  if (!make_map(&mq, a.q, a.Hq, a.total, HD, g, T) || !make_map(&mk, a.k, a.Hkv, a.total, HD, 1, BM)) return cudaErrorInvalidValue;
  CUtensorMap mpad = mq;   // (BC - T g < g heads of one token)
  if (T * g < BC && !make_map(&mpad, a.q, a.Hq, a.total, HD, BC - T * g, 1)) return cudaErrorInvalidValue;
  cudaError_t e;
  KwTable table;
  const bool by_table = a.batch <= TABLE_SEQS && (int64_t)a.n_obs * g <= 4 * BC;
  if (by_table) {
    table.first[0] = 0;
    for (int i = 0; i < a.batch; ++i)
      table.first[i + 1] = table.first[i] + (a.cu_seqlens_host[i + 1] - a.cu_seqlens_host[i] + NT * BM - 1) / (NT * BM);
  } else {
    // The whole batch is one group of the plan: sorted by work over all sequences and dealt back and forth the CTAs' loads
    // come out within 2 % of the mean (8 x 4096 tokens, 8 kv heads), where groups of a few sequences left them 15 to 40 %
    // apart.  The blocks of a (sequence, head) that run side by side still read its Q tiles through L2 together.
    e = launch_tile_plan(a.cu_seqlens, a.batch, a.max_seqlen, NT * BM, 0, plan, st);
    if (e != cudaSuccess) return e;
  }
  KwParams p{};
  p.lse = a.lse; p.weight = a.weight; p.plan = by_table ? nullptr : reinterpret_cast<const int4*>(plan); p.cu_seqlens = a.cu_seqlens; p.status = status;
  p.batch = a.batch; p.Hq = a.Hq; p.Hkv = a.Hkv; p.g = g; p.T = T; p.n_obs = a.n_obs; p.total = a.total;
  p.n_items = plan_entries * a.Hkv;
  // The same product, rounded the same way, as the prefill's: what its rounding and the truncating sums of the matrix unit add
  // to a logit is in the prefill's denominators too (D = 128), and cancels: 4096 tokens, groups of 4, logits of a standard deviation
  // of 1: 2.0e-7 off with those denominators, 1.8e-7 with exact ones; of 4: 1.9e-7 and 1.3e-6.  (A scale with the truncation's
  // mean on N(0, 1) inputs made up for does better with exact denominators, 2.5e-7 at 4, and 1.4e-6 with the prefill's.)
  p.scale_log2 = a.scale * kLog2e;
  e = ensure_dynamic_smem<key_weights_tc_kernel<HD>>(Cfg<HD>::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  e = launch_pdl(key_weights_tc_kernel<HD>, dim3(std::min(p.n_items, sm_count())), dim3(Cfg<HD>::THREADS), Cfg<HD>::SMEM_BYTES, st, mq, mpad, mk, table, p);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int key_weights_tc_rows() { return NT * BM; }

// (a group of at most 128 heads; the planner orders at most 2048 blocks a sequence; item numbers are 32-bit.  Boxes larger than
// the tensors are filled with zeros like any other rows past their end: 100 rows 5 us here, 11 on the CUDA cores.)
bool key_weights_tc_supported(const KeyWeightArgs& a, int64_t plan_entries) {
  return a.dtype == EARN_BF16 && a.Hq / a.Hkv <= BC && (a.max_seqlen + NT * BM - 1) / (NT * BM) <= 2048 &&
         plan_entries * a.Hkv < (1LL << 30);
}

cudaError_t launch_key_weights_tc(const KeyWeightArgs& a, int plan_entries, void* plan, int32_t* status_word, cudaStream_t st) {
  return a.D == 64 ? launch_hd<64>(a, plan_entries, plan, status_word, st) : launch_hd<128>(a, plan_entries, plan, status_word, st);
}

}  // namespace earn

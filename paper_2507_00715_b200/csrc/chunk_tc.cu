// Causal attention of every sequence's new tokens over its paged list, on the Blackwell tensor cores (bf16, fp32 logits,
// softmax and accumulation).
//
// A CTA (one per SM) walks its share of the work line (chunk_sched.cuh).  A row tile is 128 rows (token, query head) of one kv
// head, so that a kv head's K and V tiles of 128 keys (8 pages) serve all its query heads at once.  An item of more than one
// row tile runs two of them against the same K/V tiles; an item of at most one (a decoded token, a short chunk) runs its even
// and odd key tiles as two streams that meet in the end, so that both softmax warpgroups have work and the copies never pause.
//
//   warp 0    TMA: the pages of the K and V tiles -> shared memory (128-byte swizzle), 16 rows x 64 columns a copy, a ring that
//             runs on across items
//   warp 2    TMA: the Q tiles of the next item, as soon as the last S of the current item has read them
//   warp 3    rows behind the last key in the last page of an item: zeroed in V (a weight of zero does not undo a NaN)
//   warp 1    tcgen05.mma: S_x = Q K^T into tensor memory, O_x += P_x V with P_x read from tensor memory
//   warps 4.. one softmax warpgroup per stream x, one row per thread; the row's reference maximum is that of its first 32 visible
//             keys and raised only when a tile's sum of exponentials exceeds 2^8 (exact after the division by the row's sum)
//
// An item that is cut leaves fp32 parts; the CTA that finishes last joins them (chunk_join).  Every mbarrier wait is bounded:
// when one runs out the CTA raises its abort flag, writes EARN_ERR_TIMEOUT to the status word, waits for what it has in flight,
// frees its TMEM and returns.
#include <algorithm>
#include <type_traits>

#include "chunk_step.cuh"
#include "sm100_ptx.cuh"
#include "tc_maps.cuh"

namespace earn {
namespace {
using namespace ptx;

constexpr int BM = 128, BN = 128;
constexpr long long WAIT_LIMIT = 2000000000LL;   // about one second of SM clocks

template <int HD>
struct Cfg {
  static constexpr int TILE = 128 * HD * 2, HALF = 128 * 128;   // bytes of a tile, and of its 64-column blocks
  static constexpr int NHALF = HD / 64;
  static constexpr int NSTAGE = HD == 128 ? 4 : 8;
  static constexpr int OFF_Q = 0, OFF_RING = OFF_Q + 2 * TILE, OFF_OUT = OFF_RING + NSTAGE * TILE;
  static constexpr int OFF_ML = OFF_OUT + 8 * 4096, OFF_BAR = OFF_ML + 128 * 8;
  static constexpr int SMEM_BYTES = OFF_BAR + 768 + 1024;       // + alignment slack
  static constexpr int THREADS = 384;
  static constexpr int FULL = 0, EMPTY = FULL + NSTAGE, QFULL = EMPTY + NSTAGE, QFREE = QFULL + 2, S = QFREE + 2, P = S + 2, O = P + 2,
                       OM = O + 2, ML = OM + 1, MERGED = ML + 1, FIX = MERGED + 1, DRAIN = FIX + NSTAGE, N_BARS = DRAIN + 1;
  static_assert(8 * N_BARS + 16 + 320 <= 768, "barrier block");
};

// One item's share of this CTA.
struct Part {
  int b, kvh, head0, n_heads;   // sequence, kv head, first query head, query heads
  int tok0, tok_in, n_tok;      // first token in the batch and in the chunk, tokens
  int base, keys;               // rows in front of the chunk; keys that the item's last token sees
  int u0, n;                    // key tiles u0 .. u0 + n - 1
  bool two;                     // two row tiles; else two streams of key tiles
  bool last;                    // the item's last key tile is among them
};
__device__ __forceinline__ Part part_of(const ChunkArgs& a, const ChunkWalk& w, const ChunkSeq& q, int tile_tok) {
  const ChunkSched& s = a.sched;
  Part p;
  p.b = w.b;
  p.kvh = w.h / a.blocks;
  p.head0 = p.kvh * a.g + (w.h - p.kvh * a.blocks) * a.block_heads;
  p.n_heads = min(a.block_heads, (p.kvh + 1) * a.g - p.head0);
  p.tok_in = w.m * s.item_tok;
  p.n_tok = min(s.item_tok, q.n - p.tok_in);
  p.tok0 = q.tok0 + p.tok_in;
  p.base = q.base;
  p.keys = chunk_keys(s, q, w.m);
  const int units = chunk_units(s, q, w.m);
  p.u0 = w.off;
  p.n = (int)min((int64_t)(units - w.off), w.end - w.pos);
  p.two = p.n_tok > tile_tok;
  p.last = w.off + p.n == units;
  return p;
}
__device__ __forceinline__ void part_next(const ChunkArgs& a, ChunkWalk& w, ChunkSeq& q, const Part& p) {
  w.pos += p.n;
  if (p.last) chunk_next(a.sched, w, q);
  else w.off += p.n;
}
// Ring entries of a part, 2 n of them.  Two row tiles: K0 V0 K1 V1 ..; two streams: K0 K1 V0 K2 V1 K3 .. V(n-1), as they are
// consumed (a stream's next S follows its P V).
__device__ __forceinline__ int entry_k(const Part& p, int j) { return p.two ? 2 * j : j == 0 ? 0 : 2 * j - 1; }
__device__ __forceinline__ int entry_v(const Part& p, int j) { return p.two ? 2 * j + 1 : j == p.n - 1 ? 2 * p.n - 1 : 2 * j + 2; }
__device__ __forceinline__ void entry_at(const Part& p, int i, bool& is_v, int& j) {
  if (p.two) { is_v = i & 1; j = i >> 1; return; }
  if (i & 1) { j = (i + 1) >> 1; is_v = j >= p.n; if (is_v) j = p.n - 1; return; }
  is_v = i > 0;
  j = is_v ? (i >> 1) - 1 : 0;
}

// ---- packed fp32 pairs (one instruction for two lanes of the row) and three-input max
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c) {   // d = a * b + c
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %5};\n\t"
      "fma.rn.ftz.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float& d0, float& d1, float a0, float a1) {   // d += a
  asm("{\n\t.reg .b64 ra, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rd, {%0, %1};\n\tadd.rn.ftz.f32x2 rd, rd, ra;\n\t"
      "mov.b64 {%0, %1}, rd;\n\t}"
      : "+f"(d0), "+f"(d1) : "f"(a0), "f"(a1));
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst_smem, const CUtensorMap* map, uint32_t bar, int x, int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst_smem), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void group_sync(int x) { asm volatile("bar.sync %0, 128;" ::"r"(x + 1) : "memory"); }
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

struct TcArgs {
  ChunkArgs a;
  int tile_tok, q_box_tok;   // tokens of a row tile; tokens that a copy of Q brings
  float scale_log2;
};

template <int HD>
__global__ void __launch_bounds__(Cfg<HD>::THREADS, 1)
chunk_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TcArgs ta) {
  using C = Cfg<HD>;
  const ChunkArgs& a = ta.a;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;    // swizzled tiles need 1024-byte alignment
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base + C::OFF_Q, sRing = base + C::OFF_RING;
  const uint32_t bars = base + C::OFF_BAR;
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + C::OFF_BAR + 8 * C::N_BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + C::OFF_BAR + 8 * C::N_BARS + 8);
  int* last_part = reinterpret_cast<int*>(gen + C::OFF_BAR + 8 * C::N_BARS + 12);   // [2], behind the flag
  float2* ml1 = reinterpret_cast<float2*>(gen + C::OFF_ML);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NSTAGE; ++i) {
      mbar_init(bar(C::FULL + i), 1);
      mbar_init(bar(C::EMPTY + i), 2);   // the tensor core's reads, and warp 3
      mbar_init(bar(C::FIX + i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(C::QFULL + x), 1);
      mbar_init(bar(C::QFREE + x), 1);
      mbar_init(bar(C::S + x), 1);
      mbar_init(bar(C::P + x), 128);
      mbar_init(bar(C::O + x), 1);
    }
    mbar_init(bar(C::OM), 1);
    mbar_init(bar(C::ML), 128);
    mbar_init(bar(C::MERGED), 128);
    mbar_init(bar(C::DRAIN), 1);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;   // S_x (and P_x over it) at x * 128, O_x at (2 + x) * 128
  pdl_launch_dependents();
  pdl_wait();
  ChunkWalk w = chunk_share(a.sched, reinterpret_cast<int64_t*>(gen + C::OFF_BAR + 8 * C::N_BARS + 32));
  ChunkSeq q{};
  if (w.pos < w.end) q = chunk_seq(a.sched, w.b);
  auto wait = [&](int i, int parity) {   // warp-uniform result
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar(i), (uint32_t)parity & 1u, abort_flag, WAIT_LIMIT));
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer: K/V ring
    const int pg = lane & 7, half = lane >> 3;   // lane's page of the tile and 64-column block of it
    int e = 0;   // ring entries issued so far, over all items
    bool ok = true;
    while (w.pos < w.end && ok) {
      const Part p = part_of(a, w, q, ta.tile_tok);
      const int n_pages = (p.keys + EARN_PAGE_TOKENS - 1) / EARN_PAGE_TOKENS;
      for (int i = 0; i < 2 * p.n; ++i, ++e) {
        bool is_v;
        int j;
        entry_at(p, i, is_v, j);
        const int pages = min(n_pages - (p.u0 + j) * 8, 8), st = e % C::NSTAGE;
        bool named = false;
        int page = 0;
        if (pg < pages) page = paged_page(a.cache, p.b, (p.u0 + j) * 8 + pg, named);   // (in flight while the entry is waited for)
        if (e >= C::NSTAGE && !wait(C::EMPTY + st, (e / C::NSTAGE) - 1)) { ok = false; break; }
        if (lane == 0) mbar_expect_tx(bar(C::FULL + st), (uint32_t)max(pages, 0) * (EARN_PAGE_TOKENS * HD * 2));
        __syncwarp();
        if (pg < pages && half < C::NHALF)
          tma_load_3d(sRing + st * C::TILE + half * C::HALF + pg * (EARN_PAGE_TOKENS * 128), is_v ? &map_v : &map_k, bar(C::FULL + st),
                      half * 64, p.kvh, page * EARN_PAGE_TOKENS);
      }
      part_next(a, w, q, p);
    }
    if (*abort_flag) {
      // let the copies already in flight land before the CTA gives its shared memory back
      int none = 0;
      for (int f = max(e - C::NSTAGE, 0); f < e; ++f)
        mbar_wait_bounded(bar(C::FULL + f % C::NSTAGE), (f / C::NSTAGE) & 1, &none, WAIT_LIMIT);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------ TMA producer: Q tiles
    if (lane == 0) {
      int n[2] = {0, 0};   // tiles loaded so far
      bool ok = true;
      const uint32_t bytes = (uint32_t)(ta.q_box_tok * a.block_heads) * (HD * 2);
      while (w.pos < w.end && ok) {
        const Part p = part_of(a, w, q, ta.tile_tok);
        for (int x = 0; x < (p.two ? 2 : 1); ++x) {
          if (n[x] > 0 && !mbar_wait_bounded(bar(C::QFREE + x), (n[x] - 1) & 1, abort_flag, WAIT_LIMIT)) { ok = false; break; }
          mbar_expect_tx(bar(C::QFULL + x), bytes);
          for (int h = 0; h < C::NHALF; ++h)
            tma_load_4d(sQ + x * C::TILE + h * C::HALF, &map_q, bar(C::QFULL + x), h * 64, p.head0 - p.kvh * a.g, p.kvh,
                        p.tok0 + x * ta.tile_tok);
          ++n[x];
        }
        part_next(a, w, q, p);
      }
      if (*abort_flag) {
        int none = 0;
        for (int x = 0; x < 2; ++x)
          if (n[x] > 0) mbar_wait_bounded(bar(C::QFULL + x), (n[x] - 1) & 1, &none, WAIT_LIMIT);
      }
    }
  } else if (warp == 3) {
    // ------------------------------------------------------------------ rows of V behind the last key
    int e = 0;
    bool ok = true;
    while (w.pos < w.end && ok) {
      const Part p = part_of(a, w, q, ta.tile_tok);
      for (int i = 0; i < 2 * p.n; ++i, ++e) {
        const int st = e % C::NSTAGE;
        if (!wait(C::FULL + st, e / C::NSTAGE)) { ok = false; break; }
        const int over = p.keys % EARN_PAGE_TOKENS;
        if (p.last && i == 2 * p.n - 1 && over != 0) {   // (the last entry of a part is its last V tile)
          const int row0 = p.keys % BN, rows = EARN_PAGE_TOKENS - over;
          for (int c = lane; c < rows * 8 * C::NHALF; c += 32) {
            const int row = row0 + (c >> 3) % rows, h = (c >> 3) / rows;
            st_shared_v4(sRing + st * C::TILE + h * C::HALF + row * 128 + (c & 7) * 16, 0u, 0u, 0u, 0u);
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::FIX + st));
        }
        if (lane == 0) mbar_arrive(bar(C::EMPTY + st));
      }
      part_next(a, w, q, p);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (the warp runs the loop, lane 0 issues)
    const bool leader = lane == 0;
    constexpr uint32_t idesc_s = idesc_bf16_f32(BM, BN, 0, 0);   // Q (K-major) x K^T (K-major)
    constexpr uint32_t idesc_o = idesc_bf16_f32(BM, HD, 0, 1);   // P (TMEM) x V (MN-major)
    constexpr uint32_t desc_hi = smem_desc_hi_sw128(1024);
    const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sRing, 16), v_lo = smem_desc_lo(sRing, C::HALF);
    auto wait_full = [&](int e) { return wait(C::FULL + e % C::NSTAGE, e / C::NSTAGE); };
    // S_x = Q_y K^T with the K tile of ring entry e; free_k: nobody else reads the tile
    auto issue_s = [&](int x, int y, int e, bool free_k) {
      const uint32_t a0 = q_lo + y * (C::TILE >> 4), b0 = k_lo + (e % C::NSTAGE) * (C::TILE >> 4);
      if (leader) {
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * C::HALF + (kk & 3) * 32) >> 4;
          umma_ss_lohi(tmem + x * 128, a0 + off, desc_hi, b0 + off, desc_hi, idesc_s, kk > 0);
        }
        umma_commit(bar(C::S + x));
        if (free_k) umma_commit(bar(C::EMPTY + e % C::NSTAGE));
      }
    };
    // O_x (+)= P_x V over the pages that the tile has
    auto issue_pv = [&](int x, int e, int pages, bool first, bool free_v) {
      const uint32_t b0 = v_lo + (e % C::NSTAGE) * (C::TILE >> 4);
      if (leader) {
        if (pages >= 8) {
#pragma unroll
          for (int kk = 0; kk < BN / 16; ++kk)
            umma_ts_lohi(tmem + (2 + x) * 128, tmem + x * 128 + kk * 8, b0 + kk * (2048 >> 4), desc_hi, idesc_o, (!first || kk > 0) ? 1u : 0u);
        } else {
          for (int kk = 0; kk < pages; ++kk)
            umma_ts_lohi(tmem + (2 + x) * 128, tmem + x * 128 + kk * 8, b0 + kk * (2048 >> 4), desc_hi, idesc_o, (!first || kk > 0) ? 1u : 0u);
        }
        if (free_v) umma_commit(bar(C::EMPTY + e % C::NSTAGE));
      }
    };
    int eb = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};   // ring entry of the part's K_0; phases consumed so far
    uint32_t fix_phase = 0;                    // a bit per ring stage: warp 3 may be several items ahead, but not on one stage
    bool ok = true;
    while (w.pos < w.end && ok) {
      const Part p = part_of(a, w, q, ta.tile_tok);
      const int n = p.n, n_pages = (p.keys + EARN_PAGE_TOKENS - 1) / EARN_PAGE_TOKENS;
      // first S of both streams (the part before this one has its P V's in the queue already)
      ok = wait(C::QFULL, n_q[0]) && wait_full(eb);
      ++n_q[0];
      if (!ok) break;
      tc_fence_after();
      issue_s(0, 0, eb, !p.two);
      if (p.two) {
        ok = wait(C::QFULL + 1, n_q[1]);
        ++n_q[1];
        if (!ok) break;
        tc_fence_after();
        issue_s(1, 1, eb, true);
        if (leader && n == 1) { umma_commit(bar(C::QFREE)); umma_commit(bar(C::QFREE + 1)); }
      } else {
        if (n > 1) {
          ok = wait_full(eb + 1);
          if (!ok) break;
          tc_fence_after();
          issue_s(1, 0, eb + 1, true);
        }
        if (leader && n <= 2) umma_commit(bar(C::QFREE));
      }
      for (int j = 0; j < n && ok; ++j) {
        const int ev = eb + entry_v(p, j), pages = min(n_pages - (p.u0 + j) * 8, 8);
        const int step = p.two ? 1 : 2;                                    // tiles between two S of a stream
        const int ek = j + step < n ? eb + entry_k(p, j + step) : -1;
        for (int y = 0; y < (p.two ? 2 : 1) && ok; ++y) {
          const int x = p.two ? y : j & 1;
          ok = wait(C::P + x, n_p[x]);   // P_x written, S_x consumed
          ++n_p[x];
          if (ok && y == 0) {
            ok = wait_full(ev);
            if (ok && p.last && j == n - 1 && p.keys % EARN_PAGE_TOKENS != 0) {
              const int st = ev % C::NSTAGE;
              ok = wait(C::FIX + st, fix_phase >> st);
              fix_phase ^= 1u << st;
            }
          }
          if (!ok) break;
          tc_fence_after();
          issue_pv(x, ev, pages, j < step, !p.two || y == 1);
          if (ek >= 0) {
            if (y == 0) ok = wait_full(ek);
            if (!ok) break;
            tc_fence_after();
            issue_s(x, p.two ? x : 0, ek, !p.two || y == 1);
            if (leader && j + step == n - 1) umma_commit(bar(C::QFREE + (p.two ? x : 0)));
          } else if (leader && p.two) {
            umma_commit(bar(C::O + x));
          }
        }
      }
      if (ok && !p.two && leader) {
        umma_commit(bar(C::O));
        if (n > 1) umma_commit(bar(C::OM));
      }
      eb += 2 * n;
      part_next(a, w, q, p);
    }
    if (leader && *abort_flag) {
      int none = 0;
      umma_commit(bar(C::DRAIN));   // everything this thread issued has retired once this fires
      mbar_wait_bounded(bar(C::DRAIN), 0, &none, WAIT_LIMIT);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax warpgroup x, one row per thread
    const int x = (warp - 4) >> 2;
    const int wq = warp & 3;            // a warp may only touch TMEM lanes 32*(warp % 4) ..
    const int row = wq * 32 + lane, tok = row / a.block_heads, head = row - tok * a.block_heads;
    const uint32_t lane0 = (uint32_t)(wq * 32) << 16;
    const uint32_t t_s = tmem + lane0 + x * 128, t_o = tmem + lane0 + (2 + x) * 128;
    const float sl2 = ta.scale_log2;
    int n_s = 0, n_o = 0, n_ml = 0;   // phases consumed: S_x, O_x, merges
    bool pending = false;             // stream 1: stream 0 may still be reading what the last merge needs
    bool ok = true;
    while (w.pos < w.end && ok) {
      const Part p = part_of(a, w, q, ta.tile_tok);
      if (!p.two && x >= p.n) { part_next(a, w, q, p); continue; }   // a part of one key tile leaves stream 1 out
      const int my_tok = p.two ? x * ta.tile_tok : 0;                // first token of this stream's row tile within the item
      const int n_tok = min(ta.tile_tok, p.n_tok - my_tok);
      const bool valid = tok < n_tok && head < p.n_heads;
      const int seen = p.base + p.tok_in + my_tok + tok + 1;         // keys that the row sees
      const bool any_row = wq * 32 < n_tok * a.block_heads;          // this warp has a row
      float m_ref = -INFINITY, l0 = 0.f, l1 = 0.f;                   // -inf: no reference yet
      for (int j = p.two ? 0 : x; j < p.n; j += p.two ? 1 : 2, ++n_s) {
        ok = wait(C::S + x, n_s);
        if (!ok) break;
        tc_fence_after();
        const bool first = j < (p.two ? 1 : 2);
        if (any_row) {
          // columns visible to the row (all of them to rows that hold nothing: their values go nowhere)
          const int vis = valid ? min(max(seen - (p.u0 + j) * BN, 0), BN) : BN;
          const bool interior = __all_sync(0xffffffffu, vis == BN);
          const int n_chunks = (__reduce_max_sync(0xffffffffu, valid ? vis : 0) + 31) >> 5;   // 32-column chunks with a visible key
          uint32_t ra[32], rb[32], pk[4][16];
          // row maximum of the visible part of S_x(j), scaled into the log2 domain (a pass of its own over TMEM)
          auto row_max_all = [&]() {
            float mx = -INFINITY;
            for (int c0 = 0; c0 < n_chunks; ++c0) {
              tmem_ld_32x32(t_s + c0 * 32, ra);
              tmem_wait_ld(ra);
#pragma unroll
              for (int c = 0; c < 32; ++c) mx = fmaxf(mx, c0 * 32 + c < vis ? __uint_as_float(ra[c]) : -INFINITY);
            }
            return mx * sl2;
          };
          // P = 2^(S * scale - m_ref) as bf16 pairs (kept in registers until the reference is known to hold) and their row
          // sum, in one pass.  If the sum exceeds 2^8 some logit may have outgrown the reference, and if there is none yet the
          // first 32 columns had no finite logit: then find the tile's own maximum, raise the reference, rescale what has been
          // accumulated, and redo the pass (S_x is intact: nothing has been written over it).
          float ls0, ls1;
#pragma unroll 1
          for (int attempt = 0;; ++attempt) {
            ls0 = ls1 = 0.f;
            tmem_ld_32x32(t_s, ra);
            tmem_wait_ld(ra);
            if (first && attempt == 0) {
              float mx = -INFINITY, m1 = -INFINITY;
#pragma unroll
              for (int c = 0; c < 32; c += 4) {
                mx = max3(mx, c < vis ? __uint_as_float(ra[c]) : -INFINITY, c + 1 < vis ? __uint_as_float(ra[c + 1]) : -INFINITY);
                m1 = max3(m1, c + 2 < vis ? __uint_as_float(ra[c + 2]) : -INFINITY, c + 3 < vis ? __uint_as_float(ra[c + 3]) : -INFINITY);
              }
              m_ref = fmaxf(mx, m1) * sl2;
            }
            const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;
            // an interior tile takes a copy of the loop without a test per chunk: one block of straight-line code
            auto chunks = [&](auto interior_tag) {
              constexpr bool INTERIOR = decltype(interior_tag)::value;
#pragma unroll
              for (int c0 = 0; c0 < 4; ++c0) {
                if (INTERIOR || c0 < n_chunks) {
                  uint32_t(&cur)[32] = (c0 & 1) ? rb : ra;
                  uint32_t(&nxt)[32] = (c0 & 1) ? ra : rb;
                  if (c0 + 1 < 4 && (INTERIOR || c0 + 1 < n_chunks)) tmem_ld_32x32(t_s + (c0 + 1) * 32, nxt);
                  if (!INTERIOR) {
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                      if (c0 * 32 + c >= vis) cur[c] = 0xff800000u;   // -inf
                  }
#pragma unroll
                  for (int c = 0; c < 32; c += 2) {
                    float e0, e1;
                    fma2(e0, e1, __uint_as_float(cur[c]), __uint_as_float(cur[c + 1]), sl2, neg_m);
                    e0 = ex2(e0);
                    e1 = ex2(e1);
                    add2(ls0, ls1, e0, e1);
                    pk[c0][c >> 1] = pack_bf16(e0, e1);
                  }
                  if (c0 + 1 < 4 && (INTERIOR || c0 + 1 < n_chunks)) tmem_wait_ld(nxt);
                } else {
#pragma unroll
                  for (int c = 0; c < 16; ++c) pk[c0][c] = 0u;
                }
              }
            };
            if (interior) chunks(std::true_type{});
            else chunks(std::false_type{});
            const bool grow = valid && (!(ls0 + ls1 <= 256.f) || (m_ref == -INFINITY && vis > 0));
            if (attempt > 0 || !__any_sync(0xffffffffu, grow)) break;
            // S_x(j) was issued after the stream's last P V, so the commit that signalled it covers that too: O_x is quiescent.
            // The whole warp repeats the pass, but only the rows that asked for it take a new reference: a row's result
            // depends on its own logits alone, whatever its neighbours in the tile do.
            const float mx_all = row_max_all();
            const float mxs = grow ? mx_all : m_ref;
            const float alpha = mxs > m_ref ? ex2(m_ref - mxs) : 1.f;
            m_ref = fmaxf(m_ref, mxs);
            l0 *= alpha;
            l1 *= alpha;
            if (!first) {
#pragma unroll 1
              for (int c0 = 0; c0 < HD / 32; ++c0) {
                tmem_ld_32x32(t_o + c0 * 32, ra);
                tmem_wait_ld(ra);
#pragma unroll
                for (int c = 0; c < 32; ++c) ra[c] = __float_as_uint(__uint_as_float(ra[c]) * alpha);
                tmem_st_32x32(t_o + c0 * 32, ra);
              }
            }
          }
          l0 += ls0;
          l1 += ls1;
#pragma unroll
          for (int c0 = 0; c0 < 4; ++c0) tmem_st_32x16(t_s + c0 * 16, pk[c0]);
          tmem_wait_st();
        }
        if (pending) {   // O_1 and the numbers of the last merge are this stream's again
          ok = wait(C::MERGED, n_ml - 1);
          pending = false;
          if (!ok) break;
        }
        tc_fence_before();
        mbar_arrive(bar(C::P + x));
      }
      if (!ok) break;
      // ---- end of the part
      float l = l0 + l1, w0 = 1.f, w1 = 0.f;
      const bool merge = !p.two && p.n > 1;
      if (merge && x == 1) {
        ml1[row] = make_float2(m_ref, l);
        tc_fence_before();
        mbar_arrive(bar(C::ML));
        ++n_ml;
        pending = true;
        part_next(a, w, q, p);
        continue;
      }
      ok = wait(C::O + x, n_o++);
      if (ok && merge) ok = wait(C::OM, n_ml) && wait(C::ML, n_ml);
      if (!ok) break;
      tc_fence_after();
      if (merge) {
        ++n_ml;
        const float2 other = ml1[row];
        const float mx = fmaxf(m_ref, other.x), ref = mx == -INFINITY ? 0.f : mx;
        w0 = ex2(m_ref - ref);
        w1 = ex2(other.x - ref);
        l = l * w0 + other.y * w1;
        m_ref = mx;
      }
      const int64_t start = w.pos - w.off;
      const ChunkParts parts = chunk_parts(w, start, chunk_units(a.sched, q, w.m));
      const bool whole = parts.parts == 1;
      const float inv = !whole ? 1.f : l == 0.f ? 0.f : __frcp_rn(l);
      w0 *= inv;
      w1 *= inv;
      const int tok0 = p.tok0 + my_tok;
      const int64_t slot = (2 * (int64_t)blockIdx.x + ((int)blockIdx.x == parts.first ? 1 : 0)) * 2 + x;
      const uint32_t stage = base + C::OFF_OUT + (uint32_t)(warp - 4) * 4096;
      if (any_row) {
        uint32_t ra[32];
#pragma unroll
        for (int c0 = 0; c0 < HD / 32; ++c0) {
          tmem_ld_32x32(t_o + c0 * 32, ra);
          tmem_wait_ld(ra);
          float y[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) y[c] = __uint_as_float(ra[c]) * w0;
          if (merge) {
            tmem_ld_32x32(t_o + 128 + c0 * 32, ra);
            tmem_wait_ld(ra);
#pragma unroll
            for (int c = 0; c < 32; ++c) y[c] += __uint_as_float(ra[c]) * w1;
          }
          if (l == 0.f) {   // (nothing visible: O holds nothing)
#pragma unroll
            for (int c = 0; c < 32; ++c) y[c] = 0.f;
          }
          if (whole) {
            // 64 columns of the warp's 32 rows are staged (16-byte chunk c of row r at chunk c ^ (r % 8) of its line) and
            // written by eight lanes a row
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int ch = (c0 & 1) * 4 + c;
              st_shared_v4(stage + (uint32_t)lane * 128 + (uint32_t)((ch ^ (lane & 7)) << 4), pack_bf16(y[c * 8], y[c * 8 + 1]),
                           pack_bf16(y[c * 8 + 2], y[c * 8 + 3]), pack_bf16(y[c * 8 + 4], y[c * 8 + 5]), pack_bf16(y[c * 8 + 6], y[c * 8 + 7]));
            }
            if (c0 & 1) {
              __syncwarp();
#pragma unroll 4
              for (int i = 0; i < 8; ++i) {
                const int r = i * 4 + (lane >> 3), gr = wq * 32 + r, t = gr / a.block_heads, h = gr - t * a.block_heads;
                if (t < n_tok && h < p.n_heads) {
                  const uint4 v = ld_shared_v4(stage + (uint32_t)r * 128 + (uint32_t)(((lane & 7) ^ (r & 7)) << 4));
                  *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.o) + ((int64_t)(tok0 + t) * a.Hq + p.head0 + h) * HD +
                                            (c0 >> 1) * 64 + (lane & 7) * 8) = v;
                }
              }
              __syncwarp();
            }
          } else if (valid) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
              a.part_o[(slot * (HD / 4) + c0 * 8 + c) * BM + row] = make_float4(y[c * 4], y[c * 4 + 1], y[c * 4 + 2], y[c * 4 + 3]);
          }
        }
        if (valid && whole && a.lse != nullptr)
          a.lse[(int64_t)(p.head0 + head) * a.sched.n_tokens + tok0 + tok] = chunk_lse<true>(m_ref, l);
        if (valid && !whole) a.part_ml[slot * BM + row] = make_float2(m_ref, l);
      }
      tc_fence_before();   // the next P V over O_x is issued after this warp's next arrive on P_x
      if (merge) mbar_arrive(bar(C::MERGED));
      if (!whole) {
        __threadfence();
        group_sync(x);
        if (row == 0) {
          const int32_t at = parts.first * 2 + x;
          const bool is_last = atomicAdd(a.tickets + at, 1) == parts.parts - 1;
          if (is_last) a.tickets[at] = 0;   // for the next call
          last_part[x] = is_last;
          __threadfence();
        }
        group_sync(x);
        if (last_part[x])
          chunk_join<__nv_bfloat16, HD, BM, true>(a, parts, 2, x, row, 128, tok0, n_tok, p.head0, p.n_heads);
        group_sync(x);   // (the flag has been read)
      }
      part_next(a, w, q, p);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, (int32_t)EARN_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Q as [n_tokens, Hkv, g, D]: a copy brings a head block of `box_tok` tokens, 64 columns of it
bool make_q_map(CUtensorMap* map, const ChunkArgs& a, int box_tok) {
  auto fn = tcmap::encode_fn();
  if (fn == nullptr) return false;
  const cuuint64_t row = (cuuint64_t)a.D * 2;
  cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.g, (cuuint64_t)a.Hkv, (cuuint64_t)a.sched.n_tokens};
  cuuint64_t strides[3] = {row, row * a.g, row * a.Hq};
  cuuint32_t box[4] = {64, (cuuint32_t)a.block_heads, 1, (cuuint32_t)box_tok};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
cudaError_t launch(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st) {
  CUtensorMap mq, mk, mv;
  TcArgs ta{};
  ta.a = a;
  ta.tile_tok = p.tile_tok;
  ta.q_box_tok = std::min(p.tile_tok, a.sched.n_tokens);
  ta.scale_log2 = a.scale * kLog2e;
  const int rows = a.cache.n_pages * EARN_PAGE_TOKENS;
  if (!make_q_map(&mq, a, ta.q_box_tok) || !tcmap::make_map(&mk, a.cache.k, a.Hkv, rows, EARN_PAGE_TOKENS, HD) ||
      !tcmap::make_map(&mv, a.cache.v, a.Hkv, rows, EARN_PAGE_TOKENS, HD))
    return cudaErrorInvalidValue;
  cudaError_t e = ensure_dynamic_smem<chunk_tc_kernel<HD>>(Cfg<HD>::SMEM_BYTES);
  if (e == cudaSuccess) e = launch_pdl(chunk_tc_kernel<HD>, dim3(a.sched.grid), dim3(Cfg<HD>::THREADS), Cfg<HD>::SMEM_BYTES, st, mq, mk, mv, ta);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_chunk_tc(const ChunkArgs& a, const ChunkPlan& p, cudaStream_t st) {
  return a.D == 64 ? launch<64>(a, p, st) : launch<128>(a, p, st);
}

}  // namespace earn

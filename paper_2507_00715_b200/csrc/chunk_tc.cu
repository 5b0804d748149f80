// Causal attention of every sequence's new tokens over its paged list, on the Blackwell tensor cores (bf16, fp32 logits,
// softmax and accumulation).
//
// A CTA (one per SM) walks its share of the work line (chunk_sched.cuh) with K and V tiles of 128 keys (8 pages), each read once
// for all query heads of a kv head.  An item's rows are (token, query head); how many there are picks its form:
//
//   PAIR   more than 128 rows: two row tiles of 128 against the same K/V tiles
//   ROWS   up to 128 rows: one row tile, even and odd key tiles as two streams that meet in the end
//
// (A call of chunks of at most 16 rows, or with little work, is the other kernel's, chunk_short.cu.)
//
//   warp 0      TMA: the pages of the K and V tiles -> shared memory (128-byte swizzle), 16 rows x 64 columns a copy, a ring that
//               runs on across items
//   warp 1      what there is to do, a few parts ahead; TMA: the Q tiles of the next item, as soon as the last S of the current
//               one has read them; and the rows behind the last key in the last page of an item, zeroed in V (a weight of zero
//               does not undo a NaN)
//   warps 2, 3  tcgen05.mma, one warp per stream (row tile, or half of the key tiles): S into tensor memory, O += P V with P read
//               from tensor memory.  What a warp waits for and how long it takes to issue is hidden behind
//               the other's products: one warp for both was 1.4 times slower on long lists
//   warps 4..   softmax, two warpgroups per stream
//
// A key tile is taken in two halves of 64 keys, each with an accumulator and a warpgroup of its own, one row per
// thread, so that the tensor core has the other halves to multiply while one is in the exponentials (P lies over S: the next S
// of a half follows its P V).  With whole tiles a product of 128 x 128 costs the tensor core less (the halves read Q twice), but
// it waits more: 1152 us instead of 920 for 4096 new tokens over 12000 rows, 32/8 heads.  The reference of a row's exponentials is its largest logit among its first 32 visible keys, and
// stays: fp32 and bf16 hold 2^127, so a row needs another one only if a logit exceeds that by 44 nats or more.  If the sums tell
// that one did (or that the first keys had no finite logit), the CTA takes all its parts again, each twice: for the rows' maxima,
// and with them.  (A test per half and a rescaling of O in place, with one warpgroup per row tile, took 1.4 times as long.)
//
// The probabilities are rounded to bf16 for the product with V, the type of its instruction: outputs are off by 2.3e-3 of
// themselves, of which their own rounding makes 1.7e-3.  (A second number per probability would add the 1024 clocks of another
// product with V to a unit's 2560.)  Everything else, the row's sum included, is fp32.
//
// Measured: 4096 new tokens over 12000 rows, 32/8 heads, 850-900 us (1.05-1.1 PFLOP/s); 8 x 1024 over 16000-31000 rows 3200-3550 us (0.95-1.05,
// at the power cap); 14 chunks of 130-700 and 34 single tokens, 28/4 heads, 216 us.  A unit (256 rows x 128 keys) takes 3200 clocks,
// of which the products are 2560 and the exponentials 2048 per SM.
//
// An item that is cut leaves fp32 parts; the CTA that finishes last joins them (chunk_join), once it has nothing else to do.  Every mbarrier wait is bounded:
// when one runs out the CTA raises its abort flag, writes EARN_ERR_TIMEOUT to the status word, waits for what it has in flight,
// frees its TMEM and returns.
#include <algorithm>
#include <type_traits>

#include "chunk_part.cuh"
#include "tc_maps.cuh"

namespace earn {
namespace {

template <int HD>
struct Cfg {
  static constexpr int TILE = 128 * HD * 2, HALF = 128 * 128;   // bytes of a tile, and of its 64-column blocks
  static constexpr int NHALF = HD / 64;
  static constexpr int NSTAGE = HD == 128 ? 4 : 8;
  static constexpr int OFF_Q = 0, OFF_RING = OFF_Q + 2 * TILE, RING_END = OFF_RING + NSTAGE * TILE;
  static constexpr int OFF_REF = RING_END;                                             // references [stream][row]
  static constexpr int OFF_SUM = OFF_REF + 2 * 128 * 4;                                // sums [parity][stream][half][row]
  static constexpr int OFF_MAX = OFF_SUM + 2 * 2 * 2 * 128 * 4;                        // maxima [stream][half][row]
  static constexpr int OFF_SUM1 = OFF_MAX + 2 * 2 * 128 * 4;                           // stream 1's sums [half][row] for a merge
  static constexpr int OFF_CUT = OFF_SUM1 + 2 * 128 * 4;                               // parts of items that are cut [stream][2]
  static constexpr int OFF_SEQ = OFF_CUT + 4 * 64;                                          // the sequences
  static constexpr int OFF_PART = OFF_SEQ + kChunkTable * (int)sizeof(ChunkSeq), OFF_BAR = OFF_PART + 4 * 64;
  static constexpr int THREADS = 32 * 20;
  static constexpr int FULL = 0, EMPTY = FULL + NSTAGE, QFULL = EMPTY + NSTAGE, QFREE = QFULL + 2, S = QFREE + 2, P = S + 4, O = P + 4,
                       OM = O + 2, ML = OM + 1, MERGED = ML + 1, FIX = MERGED + 1, DRAIN = FIX + NSTAGE, PARTFULL = DRAIN + 2,
                       PARTFREE = PARTFULL + 4, REFS = PARTFREE + 4, SUMS = REFS + 2, DONE = SUMS + 2,
                       OFREE = DONE + 1, N_BARS = OFREE + 2;
  static constexpr int SMEM_BYTES = OFF_BAR + (8 * N_BARS + 48 + 127) / 128 * 128 + 1024;   // + alignment slack
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of an SM");
};

constexpr float SUM_LIMIT = 1.8446744e19f;   // 2^64: sums up to here leave O's below 2^64 |v|

// Ring entries of a part, 2 n of them.  PAIR: K0 V0 K1 V1 ..; two streams: K0 K1 V0 K2 V1 K3 .. V(n-1), as they are consumed (a
// stream's next S follows its P V).
__device__ __forceinline__ int entry_k(const Part& p, int j) { return p.form() == PAIR ? 2 * j : j == 0 ? 0 : 2 * j - 1; }
__device__ __forceinline__ int entry_v(const Part& p, int j) { return p.form() == PAIR ? 2 * j + 1 : j == p.n - 1 ? 2 * p.n - 1 : 2 * j + 2; }
__device__ __forceinline__ void entry_at(const Part& p, int i, bool& is_v, int& j) {
  if (p.form() == PAIR) { is_v = i & 1; j = i >> 1; return; }
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
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c0, float c1) {   // d = a * b + c
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %6};\n\t"
      "fma.rn.ftz.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c0), "f"(c1));
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
__device__ __forceinline__ void tmem_ld_16(uint32_t taddr, uint32_t (&r)[16]) {   // 32 lanes x 16 columns, to be waited for
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16]) {
  tmem_ld_16(taddr, r);
  tmem_wait_16(r);
}
__device__ __forceinline__ void tmem_st_8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
constexpr float NO_REF = 3.0e38f;   // added to a logit that has no reference yet: 2^(that) is inf unless the logit is -inf

// The same instructions as in sm100_ptx.cuh, issued by one elected lane of a converged warp, so that the descriptors stay
// warp-uniform arithmetic (a branch on the lane around them cost 1.1 times the time on long lists).
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
               "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void st_global_32b(void* at, const uint32_t (&v)[8]) {   // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ float lds(uint32_t at) { float v; asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory"); return v; }
__device__ __forceinline__ void sts(uint32_t at, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }

struct TcArgs {
  ChunkArgs a;
  int tile_tok, q_box_tok;   // tokens of a row tile; tokens that a copy of Q brings
  float scale_log2;
};

// Phases that a warpgroup has consumed: S, O, references, sums, merges of the streams.
struct Phases {
  int s, o, ref, sum, ml;
  bool pending;   // stream 1: stream 0 may still be reading what the last merge needs
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
  volatile int* redo = reinterpret_cast<volatile int*>(gen + C::OFF_BAR + 8 * C::N_BARS + 12);       // a sum left the range: all parts again
  volatile int* last_part = reinterpret_cast<volatile int*>(gen + C::OFF_BAR + 8 * C::N_BARS + 16);  // [stream][2]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NSTAGE; ++i) {
      mbar_init(bar(C::FULL + i), 1);
      mbar_init(bar(C::EMPTY + i), 3);   // both streams, warp 1
      mbar_init(bar(C::FIX + i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(C::QFULL + x), 1);
      mbar_init(bar(C::QFREE + x), 2 - x);   // both streams see the first Q tile, the second one only stream 1
      mbar_init(bar(C::O + x), 1);
      mbar_init(bar(C::REFS + x), 4);
      mbar_init(bar(C::SUMS + x), 8);
      mbar_init(bar(C::OFREE + x), 8);   // the warps that read O_x: its stream's, or stream 0's where the streams meet
    }
    for (int i = 0; i < 4; ++i) {   // stream, half of the key tile
      mbar_init(bar(C::S + i), 1);
      mbar_init(bar(C::P + i), 4);   // (one lane a warp)
    }
    mbar_init(bar(C::OM), 1);
    mbar_init(bar(C::ML), 8);
    mbar_init(bar(C::MERGED), 8);
    mbar_init(bar(C::DONE), 16);
    mbar_init(bar(C::DRAIN), 1);
    mbar_init(bar(C::DRAIN + 1), 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(C::PARTFULL + i), 1);
      mbar_init(bar(C::PARTFREE + i), 19);   // warps 0, 2, 3 and the softmax warps
    }
    *abort_flag = 0;
    *redo = 0;
    fence_barrier_init();
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  if (warp == 2) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;   // S_x (and P_x over it) at x * 128, O_x at (2 + x) * 128
  pdl_launch_dependents();
  pdl_wait();
  if (!chunk_many(a.sched, a.split)) {   // (the call is the other kernel's)
    if (warp == 2) tmem_dealloc(tmem, 512);
    return;
  }
  ChunkSched sched = a.sched;
  ChunkWalk w = chunk_share(sched, reinterpret_cast<int4*>(gen), reinterpret_cast<ChunkSeq*>(gen + C::OFF_SEQ));
  fence_async_smem();   // (the copies that come next land where the shares' scratch was)
  __syncthreads();
  auto wait = [&](int i, int parity) { return warp_wait(bar(i), parity, abort_flag); };

  auto get_part = [&](int k, Part& p) { return take_part(gen + C::OFF_PART, bar(C::PARTFULL), bar(C::PARTFREE), k, abort_flag, p); };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer: K/V ring
    const int pg = lane & 7, half = lane >> 3;   // lane's page of the tile and 64-column block of it
    int e = 0;   // ring entries issued so far, over all parts
    bool ok = true;
    Part p;
    for (int k = 0; ok && get_part(k, p); ++k) {
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
    }
    if (*abort_flag) {
      // let the copies already in flight land before the CTA gives its shared memory back
      int none = 0;
      for (int f = max(e - C::NSTAGE, 0); f < e; ++f)
        mbar_wait_bounded(bar(C::FULL + f % C::NSTAGE), (f / C::NSTAGE) & 1, &none, WAIT_LIMIT);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ parts; TMA producer: Q tiles; rows of V behind the last key
    const ChunkWalk begin = w;
    ChunkSeq q{};
    if (w.pos < w.end) q = chunk_seq(sched, w.b);
    int e = 0, n_q[2] = {0, 0}, made = 0;   // ring entries passed, Q tiles loaded, parts handed out so far
    bool ok = true, more = true;
    int pass = FAST;
    Part again{};   // EXACT: the part whose maxima were just asked for
    const uint32_t bytes = (uint32_t)(ta.q_box_tok * a.block_heads) * (HD * 2);
    for (int k = 0; ok; ++k) {
      auto hand_out = [&](int upto) {
        while (more && made <= upto) {
          Part fresh;
          if (pass == EXACT && again.n > 0) {
            fresh = again;
            fresh.kind += 4 * (EXACT - MAXIMA);
            again.n = 0;
          } else {
            fresh = next_part(a, sched, w, q, ta.tile_tok, pass == FAST ? FAST : MAXIMA);
            if (fresh.n > 0 && pass == EXACT) again = fresh;
            if (fresh.n < 0) {
              more = false;
              if (pass == FAST) fresh.n = 0;   // (this warp goes on once it has come to it)
            }
          }
          if (!give_part(gen + C::OFF_PART, bar(C::PARTFULL), bar(C::PARTFREE), made, abort_flag, fresh)) return false;
          ++made;
        }
        return true;
      };
      ok = hand_out(k);
      if (!ok) break;
      const Part p = *reinterpret_cast<const Part*>(gen + C::OFF_PART + (k & 3) * 64);
      if (p.n < 0) break;
      if (p.n == 0) {   // every softmax warp has come to the end of its parts: do they have to be taken again?
        ok = wait(C::DONE, 0);
        pass = EXACT;
        if (*redo != 0) {
          w = begin;
          if (w.pos < w.end) q = chunk_seq(sched, w.b);
        }
        more = true;
        continue;
      }
      for (int x = 0; x < (p.form() == PAIR ? 2 : 1); ++x) {
        if (n_q[x] > 0 && !wait(C::QFREE + x, n_q[x] - 1)) { ok = false; break; }
        if (lane == 0) {
          mbar_expect_tx(bar(C::QFULL + x), bytes);
          for (int h = 0; h < C::NHALF; ++h)
            tma_load_4d(sQ + x * C::TILE + h * C::HALF, &map_q, bar(C::QFULL + x), h * 64, p.head0 - p.kvh * a.g, p.kvh,
                        p.tok0 + x * ta.tile_tok);
        }
        ++n_q[x];
      }
      ok = ok && hand_out(k + 2);   // two parts ahead (four places: this warp reads its own there)
      for (int i = 0; i < 2 * p.n && ok; ++i, ++e) {
        const int st = e % C::NSTAGE;
        ok = wait(C::FULL + st, e / C::NSTAGE);
        if (!ok) break;
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
    }
    if (*abort_flag) {
      int none = 0;
      for (int x = 0; x < 2; ++x)
        if (n_q[x] > 0) mbar_wait_bounded(bar(C::QFULL + x), (n_q[x] - 1) & 1, &none, WAIT_LIMIT);
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------------ MMA issuer of stream x
    const int x = warp - 2;
    constexpr uint32_t idesc_s = idesc_bf16_f32(BM, BN / 2, 0, 0);   // Q (K-major) x half a K tile^T (K-major)
    constexpr uint32_t idesc_o = idesc_bf16_f32(BM, HD, 0, 1);       // P (TMEM) x V (MN-major)
    constexpr uint32_t desc_hi = smem_desc_hi_sw128(1024);
    const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sRing, 16), v_lo = smem_desc_lo(sRing, C::HALF);
    const uint32_t t_s = tmem + x * 128, t_o = tmem + (2 + x) * 128;
    auto free_entry = [&](int e) { mma_commit(bar(C::EMPTY + e % C::NSTAGE)); };
    // S of half b of a row tile: Q_y times keys 64 b .. of the K tile of ring entry e
    auto issue_s = [&](int b, int y, int e) {
      const uint32_t a0 = q_lo + y * (C::TILE >> 4), b0 = k_lo + ((e % C::NSTAGE) * C::TILE + b * (64 * 128) >> 4);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk) {
        const uint32_t off = ((kk >> 2) * C::HALF + (kk & 3) * 32) >> 4;
        mma_ss(t_s + b * 64, a0 + off, b0 + off, desc_hi, idesc_s, kk > 0);
      }
      mma_commit(bar(C::S + 2 * x + b));
    };
    // O (+)= P V over the pages that half b of the tile has
    auto issue_pv = [&](int b, int e, int pages, bool first) {
      const uint32_t b0 = v_lo + ((e % C::NSTAGE) * C::TILE + b * (64 * 128) >> 4);
      const uint32_t more = first ? 0u : 1u;
      if (pages >= 4 * b + 4) {   // (without a test per product: the tests cost as much as the products)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(t_o, t_s + b * 64 + kk * 8, b0 + kk * (2048 >> 4), desc_hi, idesc_o, kk > 0 ? 1u : more);
      } else {
#pragma unroll 1
        for (int kk = 0; 4 * b + kk < pages; ++kk) mma_ts(t_o, t_s + b * 64 + kk * 8, b0 + kk * (2048 >> 4), desc_hi, idesc_o, kk > 0 ? 1u : more);
      }
    };
    int eb = 0, n_q = 0, n_q0 = 0;   // ring entry of the part's K_0; parts with a second Q tile, and all
    int n_o = 0;                     // parts that had their sums in O_x
    int filled = 0;                  // ring entries waited for
    uint32_t p_phase = 0;            // a bit per P barrier
    uint32_t fix_phase = 0;          // a bit per ring stage: warp 1 may be several items ahead, but not on one stage
    auto wait_p = [&](int b) {
      const bool done = wait(C::P + 2 * x + b, p_phase >> b);
      p_phase ^= 1u << b;
      return done;
    };
    bool ok = true;
    Part p;
    for (int k = 0; ok && get_part(k, p); ++k) {
      if (p.n == 0) continue;
      const int n = p.n, n_pages = (p.keys + EARN_PAGE_TOKENS - 1) / EARN_PAGE_TOKENS;
      const int stride = p.form() == PAIR ? 1 : 2, y = p.form() == PAIR ? x : 0, j0 = p.form() == PAIR ? 0 : x;
      const bool fixed = p.last && p.keys % EARN_PAGE_TOKENS != 0;   // the last V tile is one that warp 1 works on
      const int fix_st = (eb + 2 * n - 1) % C::NSTAGE;
      // Every entry is waited for, the other stream's too (and handed on at once): a barrier's parity tells the phase only to
      // those who leave none out.
      auto wait_full = [&](int e) {
        for (; filled <= e; ++filled) {
          const int st = filled % C::NSTAGE;
          if (!wait(C::FULL + st, filled / C::NSTAGE)) return false;
          bool is_v;
          int j;
          entry_at(p, filled - eb, is_v, j);
          if (p.form() != PAIR && (j & 1) != x && lane == 0) mbar_arrive(bar(C::EMPTY + st));
        }
        return true;
      };
      ok = wait(C::QFULL, n_q0);
      if (ok && (y == 1 || j0 >= n) && lane == 0) mbar_arrive(bar(C::QFREE));   // (seen, but not read)
      if (ok && y == 1) ok = wait(C::QFULL + 1, n_q);
      if (!ok) break;
      if (j0 < n) {
        ok = wait_full(eb + entry_k(p, j0));
        if (!ok) break;
        tc_fence_after();
        auto wait_v = [&](int j) { return wait_full(eb + entry_v(p, j)) && (!fixed || j + 1 < n || wait(C::FIX + fix_st, fix_phase >> fix_st)); };
        auto pages_of = [&](int j) { return min(n_pages - (p.u0 + j) * 8, 8); };
        auto free_q = [&]() { mma_commit(bar(C::QFREE + y)); };   // the stream's last S has been issued
        {
          issue_s(0, y, eb + entry_k(p, j0));
          issue_s(1, y, eb + entry_k(p, j0));
          free_entry(eb + entry_k(p, j0));
          if (j0 + stride >= n) free_q();
          if (n_o > 0) ok = wait(C::OFREE + x, n_o - 1);   // the first P V overwrites what both halves' warps read at the last part's end
          ++n_o;
          for (int j = j0; j < n && ok; j += stride) {
            const int ev = eb + entry_v(p, j), ek = eb + entry_k(p, j + stride), pages = pages_of(j);
            const bool more = j + stride < n;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              ok = wait_p(b) && (b > 0 || wait_v(j));   // P written, S consumed
              if (!ok) break;
              tc_fence_after();
              issue_pv(b, ev, pages, j == j0 && b == 0);
              if (b == 1) free_entry(ev);
              if (more) {
                if (b == 0) ok = wait_full(ek);
                if (!ok) break;
                tc_fence_after();
                issue_s(b, y, ek);
                if (b == 1) {
                  free_entry(ek);
                  if (j + 2 * stride >= n) free_q();
                }
              }
            }
          }
        }
        if (ok) mma_commit(bar(p.form() == PAIR || x == 0 ? C::O + x : C::OM));
      }
      ok = ok && wait_full(eb + 2 * n - 1);
      ++n_q0;
      if (p.form() == PAIR) ++n_q;
      if (fixed) fix_phase ^= 1u << fix_st;
      eb += 2 * n;
    }
    if (*abort_flag) {
      int none = 0;
      mma_commit(bar(C::DRAIN + x));   // everything this warp issued has retired once this fires
      mbar_wait_bounded(bar(C::DRAIN + x), 0, &none, WAIT_LIMIT);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax: stream x, half b of its key tiles
    const int x = (warp - 4) >> 3, b = ((warp - 4) >> 2) & 1;
    const int wq = warp & 3;            // a warp may only touch TMEM lanes 32*(warp % 4) ..
    const int row = wq * 32 + lane;
    const float sl2 = ta.scale_log2;
    Phases n{};
    Part* cuts = reinterpret_cast<Part*>(gen + C::OFF_CUT + x * 128);   // (written by the first half's threads)
    int n_cuts = 0;
    bool ok = true, again = false;
    Part p;
    {
      const int per_head = 65536 / a.block_heads + 1;   // row * per_head >> 16 = row / block_heads for rows below 128
      const int tok = row * per_head >> 16, head = row - tok * a.block_heads;
      const uint32_t lane0 = (uint32_t)(wq * 32) << 16;
      const uint32_t t_s = tmem + lane0 + x * 128 + b * 64, t_o = tmem + lane0 + (2 + x) * 128 + b * (HD / 2);
      const uint32_t refs = base + C::OFF_REF + (uint32_t)row * 4, sums = base + C::OFF_SUM + (uint32_t)row * 4, maxima = base + C::OFF_MAX + (uint32_t)row * 4, sums1 = base + C::OFF_SUM1 + (uint32_t)row * 4;
      for (int k = 0; ok && get_part(k, p); ++k) {
        if (p.n == 0) {   // the end of a pass
          warp_arrive(bar(C::DONE));
          again = true;
          continue;
        }
        if (again) {      // all parts once more
          n_cuts = 0;
          again = false;
        }
        const bool pair = p.form() == PAIR, merge = !pair && p.n > 1;
        if (!pair && x >= p.n) continue;   // a part of one key tile leaves stream 1 out
        if (n.pending) {                   // stream 0 has read what the last merge needs
          n.pending = false;
          ok = wait(C::MERGED, n.ml - 1);
          if (!ok) break;
        }
        const int stride = pair ? 1 : 2, my_tok = pair ? x * ta.tile_tok : 0, pass = p.pass();
        const int n_tok = min(ta.tile_tok, p.n_tok - my_tok);
        const bool valid = tok < n_tok && head < p.n_heads;
        const int seen = p.base + p.tok_in + my_tok + tok + 1;         // keys that the row sees
        const bool any_row = wq * 32 < n_tok * a.block_heads;          // this warp has a row
        const int seen_least = __reduce_min_sync(0xffffffffu, valid ? seen : INT32_MAX), seen_most = __reduce_max_sync(0xffffffffu, valid ? seen : 0);
        float neg_m = NO_REF, l0 = 0.f, l1 = 0.f, top = -INFINITY;
        const int j0 = pair ? 0 : x;
        for (int j = j0; j < p.n; j += stride) {
          ok = wait(C::S + 2 * x + b, n.s++);
          if (!ok) break;
          tc_fence_after();
          const int key0 = (p.u0 + j) * BN + b * 64;
          // columns visible to the row (all of them to rows that hold nothing: their values go nowhere)
          const int vis = valid ? min(max(seen - key0, 0), 64) : 64;
          if (j == j0) {   // the row's reference: from the first half's first 32 columns, or the maxima of the pass before
            if (b == 0) {
              if (pass == EXACT) {
                neg_m = -fmaxf(lds(maxima + x * 1024), lds(maxima + x * 1024 + 512));
              } else if (any_row) {
                float mx = -INFINITY;
#pragma unroll
                for (int c0 = 0; c0 < 32; c0 += 16) {
                  uint32_t s[16];
                  tmem_ld_32x16(t_s + c0, s);
#pragma unroll
                  for (int c = 0; c < 16; c += 2)
                    mx = max3(mx, c0 + c < vis ? __uint_as_float(s[c]) : -INFINITY, c0 + c + 1 < vis ? __uint_as_float(s[c + 1]) : -INFINITY);
                }
                neg_m = -mx * sl2;
              }
              if (neg_m == INFINITY) neg_m = NO_REF;   // (no finite logit)
              sts(refs + x * 512, neg_m);
              warp_arrive(bar(C::REFS + x));
            } else {
              ok = wait(C::REFS + x, n.ref++);
              if (!ok) break;
              neg_m = lds(refs + x * 512);
            }
          }
          if (any_row) {
            // P = 2^(S * scale - reference) as bf16 pairs over the first columns of S, and the row's sum, 16 columns at a time.  A
            // half that all rows see whole takes a copy without a test per column.
            auto half = [&](auto interior) {
              uint32_t s[2][16];
              tmem_ld_16(t_s, s[0]);
              tmem_wait_16(s[0]);
#pragma unroll
              for (int c0 = 0; c0 < 4; ++c0) {
                uint32_t(&cur)[16] = s[c0 & 1];
                if (c0 < 3) tmem_ld_16(t_s + (c0 + 1) * 16, s[(c0 + 1) & 1]);
                if (!decltype(interior)::value) {
#pragma unroll
                  for (int c = 0; c < 16; ++c)
                    if (c0 * 16 + c >= vis) cur[c] = 0xff800000u;   // -inf
                }
                uint32_t pk[8];
#pragma unroll
                for (int c = 0; c < 16; c += 2) {
                  float e0, e1;
                  fma2(e0, e1, __uint_as_float(cur[c]), __uint_as_float(cur[c + 1]), sl2, neg_m, neg_m);
                  e0 = ex2(e0);
                  e1 = ex2(e1);
                  add2(l0, l1, e0, e1);
                  pk[c >> 1] = pack_bf16(e0, e1);
                }
                if (c0 < 3) tmem_wait_16(s[(c0 + 1) & 1]);
                tmem_st_8(t_s + c0 * 8, pk);
              }
              tmem_wait_st();
            };
            if (pass == MAXIMA) {
#pragma unroll 1
              for (int c0 = 0; c0 < 64; c0 += 16) {
                uint32_t s[16];
                tmem_ld_32x16(t_s + c0, s);
#pragma unroll
                for (int c = 0; c < 16; ++c)
                  if (c0 + c < vis) top = fmaxf(top, __uint_as_float(s[c]));
              }
            } else if (seen_least >= key0 + 64) {
              half(std::true_type{});
            } else {
              half(std::false_type{});
            }
          }
          tc_fence_before();
          warp_arrive(bar(C::P + 2 * x + b));
        }
        if (!ok) break;
        // ---- end of the part: the halves' sums meet, and the streams'
        const uint32_t mine = merge && x == 1 ? sums1 : sums + (uint32_t)(((n.sum & 1) * 2 + x) * 1024);
        sts(mine + b * 512, l0 + l1);
        if (pass == MAXIMA) sts(maxima + x * 1024 + b * 512, top * sl2);
        if (merge && x == 1) {
          tc_fence_before();
          warp_arrive(bar(C::ML));
          ++n.ml;
          n.pending = true;
          continue;
        }
        warp_arrive(bar(C::SUMS + x));
        ok = wait(C::SUMS + x, n.sum++) && wait(C::O + x, n.o++);
        if (ok && merge) ok = wait(C::OM, n.ml) && wait(C::ML, n.ml);
        if (!ok) break;
        tc_fence_after();
        float l = lds(mine) + lds(mine + 512), m_ref = neg_m == NO_REF ? -INFINITY : -neg_m, w0 = 1.f, w1 = 0.f;
        bool fits = l <= SUM_LIMIT;
        if (merge) {
          ++n.ml;
          const float other = lds(sums1) + lds(sums1 + 512), neg1 = lds(refs + 512), m1 = neg1 == NO_REF ? -INFINITY : -neg1;
          fits = fits && other <= SUM_LIMIT;
          const float mx = fmaxf(m_ref, m1), ref = mx == -INFINITY ? 0.f : mx;
          w0 = ex2(m_ref - ref);
          w1 = ex2(m1 - ref);
          l = l * w0 + other * w1;
          m_ref = mx;
        }
        if (pass == FAST && valid && !fits) *redo = 1;
        const bool whole = p.parts == 1;
        if (any_row && pass != MAXIMA) {
          const float inv = !whole ? 1.f : l == 0.f ? 0.f : __frcp_rn(l);
          w0 *= inv;
          w1 *= inv;
          const int64_t slot = part_slot(p, x);
          const int at_tok = p.tok0 + my_tok + tok;
          __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(a.o) + ((int64_t)at_tok * a.Hq + p.head0 + head) * HD + b * (HD / 2);
          const bool by32 = (reinterpret_cast<uintptr_t>(a.o) & 31) == 0;
#pragma unroll
          for (int c0 = 0; c0 < HD / 32; ++c0) {   // this half's columns of O, 16 at a time
            uint32_t s0[16], s1[16];
            float y[16];
            tmem_ld_32x16(t_o + c0 * 16, s0);
            if (merge) tmem_ld_32x16(t_o + 128 + c0 * 16, s1);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              y[c] = __uint_as_float(s0[c]) * w0;
              if (merge) y[c] += __uint_as_float(s1[c]) * w1;
              if (l == 0.f) y[c] = 0.f;   // (nothing visible: O holds nothing)
            }
            if (valid && whole) {
              uint32_t v[8];
#pragma unroll
              for (int c = 0; c < 8; ++c) v[c] = pack_bf16(y[2 * c], y[2 * c + 1]);
              if (by32) {
                st_global_32b(o + c0 * 16, v);
              } else {
                *reinterpret_cast<uint4*>(o + c0 * 16) = make_uint4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint4*>(o + c0 * 16 + 8) = make_uint4(v[4], v[5], v[6], v[7]);
              }
            } else if (valid) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
                a.part_o[(slot * (HD / 4) + b * (HD / 8) + c0 * 4 + c) * BM + row] = make_float4(y[c * 4], y[c * 4 + 1], y[c * 4 + 2], y[c * 4 + 3]);
            }
          }
          if (b == 0 && valid) {
            if (!whole) a.part_ml[slot * BM + row] = make_float2(m_ref, l);
            else if (a.lse != nullptr) a.lse[(int64_t)(p.head0 + head) * a.sched.n_tokens + at_tok] = chunk_lse<true>(m_ref, l);
          }
        }
        tc_fence_before();
        warp_arrive(bar(C::OFREE + x));   // this warp has read O_x: the next part's first P V waits for all of them
        if (merge) {
          warp_arrive(bar(C::OFREE + 1));
          warp_arrive(bar(C::MERGED));
        }
        if (!whole && pass != MAXIMA) {
          if (b == 0 && row == 0) cuts[n_cuts] = p;
          ++n_cuts;
        }
      }
    }
    // ---- items that are cut: both warpgroups have written their columns of the parts
    warp_arrive(bar(C::DONE));
    if (ok && n_cuts > 0 && wait(C::DONE, 1)) {   // (the other stream is through as well: the join's weights go over Q and the ring)
      auto sync = [&]() {
        warp_arrive(bar(C::SUMS + x));
        return wait(C::SUMS + x, n.sum++);
      };
      join_cuts<HD, false>(a, cuts, n_cuts, ta.tile_tok, x, b * 128 + row, last_part + 2 * x, reinterpret_cast<float*>(gen + x * (128 * 160 * 4)), sync);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, (int32_t)EARN_ERR_TIMEOUT);
  if (warp == 2) {
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
  // An item of two row tiles takes 7 to 10 thousand clocks besides its key tiles, 3.2 thousand each; one of a single row tile,
  // whose streams meet while the next part begins, next to nothing.  (48 mixed sequences: 218.5 us without, 215.7 with 2.)
  ta.a.sched.item_cost = kItemCost;
  ta.a.sched.free_tok = p.tile_tok;
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

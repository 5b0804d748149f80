// Rotary positions: pairs of a head's first `rot` elements are turned by angle f_i * position and scaled by the amplitude,
//   y_a = A (x_a cos - x_b sin),  y_b = A (x_a sin + x_b cos),   pair i = (i, i + rot/2), or (2i, 2i + 1) interleaved;
// the rest of the head is copied.  The gradient is the transposed turn (sin negated).  In the append form the rows of K go,
// turned, and those of V, as they are, to their slots in the page pool.
//
// Bound by HBM: every row is read and written once.  Angles cost a token rot/2 sines and cosines, shared by all its heads:
// the product position * f_i is taken and reduced to turns in 64 bits (a 32-bit product is off by 0.06 rad at position 10^6),
// the remainder's sine and cosine in 32.  They go to shared memory, from where the threads take them, eight pairs at a time.
// 65536 tokens of 32/8 heads of 128: 233 us, 5.8 TB/s of a copy's 6.55; 8191 tokens of 28/4 heads appended: 26 us, 5.8 TB/s; 64
// tokens: 2.5 us, a launch.
#include <algorithm>

#include "chunk_step.cuh"

namespace earn {
namespace {

constexpr int MAX_TOKENS = 8;

enum Form { HALF, INTERLEAVED, STAGED };   // STAGED: half layout whose second half does not start on a 16-byte vector

template <typename T> struct Vec { static constexpr int N = 16 / (int)sizeof(T); };

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float (&x)[Vec<T>::N]) {
  const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) x[i] = (float)e[i];
}
template <typename T>
__device__ __forceinline__ uint4 packed(const float (&x)[Vec<T>::N]) {
  uint4 w;
  T* e = reinterpret_cast<T*>(&w);
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) e[i] = (T)x[i];
  return w;
}

// One token's rows: where head h (Q heads, K heads, V heads, counted through) is read and written.  dst null: not written.
struct Row {
  const char* src;
  char* dst;
  bool turn;
};
__device__ __forceinline__ Row row_of(const RopeArgs& a, int tok, int h, int slot, int head_bytes) {
  Row r;
  if (h < a.Hq) {
    r.src = a.q + tok * a.q_stride + (int64_t)h * head_bytes;
    r.dst = a.q_out + ((int64_t)tok * a.Hq + h) * head_bytes;
    r.turn = true;
    return r;
  }
  h -= a.Hq;
  const bool is_v = h >= a.Hkv;
  if (is_v) h -= a.Hkv;
  r.turn = !is_v;
  r.src = is_v ? a.v + tok * a.v_stride + (int64_t)h * head_bytes : a.k + tok * a.k_stride + (int64_t)h * head_bytes;
  if (a.slots != nullptr) {
    const bool ok = slot >= 0 && slot < a.cache.n_pages * EARN_PAGE_TOKENS;
    char* base = is_v ? a.cache.v : a.cache.k;
    r.dst = ok ? base + ((int64_t)slot * a.Hkv + h) * head_bytes : nullptr;
  } else {
    r.dst = a.k_out + ((int64_t)tok * a.Hkv + h) * head_bytes;
  }
  return r;
}

// A block takes `tokens` tokens and `per_block` of their heads, as one list of units.  A thread's first two units are on their
// way while the angles are worked out.  Loads and stores are marked as streaming: the rows are read once, and what is written is
// read by another kernel or not soon (65536 tokens 237 us without, 233 with; the attention behind an append of 8 x 1024 tokens is
// as fast).
template <typename T, int D, int FORM, int THREADS>
__global__ void __launch_bounds__(THREADS) rope_kernel(RopeArgs a, int heads, int head_from, int per_block, int tokens) {
  constexpr int N = Vec<T>::N, HEAD_BYTES = D * (int)sizeof(T);
  constexpr int UNITS = FORM == HALF ? D / (2 * N) : D / N;   // HALF: a unit is two vectors, a pair's halves or two that are copied
  constexpr int VECS = FORM == HALF ? 2 : 1, AHEAD = 2;
  __shared__ float2 cs[MAX_TOKENS][D / 2];
  __shared__ int place[MAX_TOKENS][2];   // position, slot
  extern __shared__ uint4 rows[];        // STAGED: the rows
  const int t = threadIdx.x, tok0 = blockIdx.x * tokens, half = a.rot / 2;
  head_from += (int)blockIdx.y * per_block;   // this block's heads
  heads = min(per_block, heads - (int)blockIdx.y * per_block);
  tokens = min(tokens, a.n_tokens - tok0);
  const int units = heads * UNITS, all = tokens * units, turned = half / N;
  pdl_launch_dependents();
  pdl_wait();
  if (t < tokens) {
    place[t][0] = a.positions[tok0 + t];
    place[t][1] = a.slots != nullptr ? a.slots[tok0 + t] : -1;
  }
  // unit i of the block: its token, head, number; HALF: pairs' units first (vectors u and u + half / N), then the copied ones, two
  // by two behind the turned share
  auto load = [&](int i, uint4 (&w)[VECS]) {
    const int k = tokens == 1 ? 0 : i / units, r = i - k * units, u = r % UNITS;
    const uint4* src = reinterpret_cast<const uint4*>(row_of(a, tok0 + k, head_from + r / UNITS, -1, HEAD_BYTES).src);
    if constexpr (FORM == HALF) {
      w[0] = __ldcs(src + (u < turned ? u : 2 * u));
      w[1] = __ldcs(src + (u < turned ? u + turned : 2 * u + 1));
    } else {
      w[0] = __ldcs(src + u);
    }
  };
  uint4 ahead[AHEAD][VECS];
#pragma unroll
  for (int n = 0; n < AHEAD; ++n)
    if (t + n * THREADS < all) load(t + n * THREADS, ahead[n]);
  for (int i = t; i < tokens * half; i += THREADS) {
    const int k = i / half, p = i - k * half;
    const double turns = (double)a.positions[tok0 + k] * a.freq[p] * 0.15915494309189533577, rest = turns - rint(turns);   // 1 / (2 pi)
    float sn, cn;
    const float by = (float)(2.0 * rest), lost = (float)(2.0 * rest - (double)by) * 3.14159265f;
    sincospif(by, &sn, &cn);
    // (what the angle lost to 32 bits is put back to first order)
    cs[k][p] = make_float2(a.amplitude * fmaf(-lost, sn, cn), a.sign * a.amplitude * fmaf(lost, cn, sn));
  }
  if constexpr (FORM == STAGED) {
#pragma unroll
    for (int n = 0; n < AHEAD; ++n)
      if (t + n * THREADS < all) rows[t + n * THREADS] = ahead[n][0];
    for (int i = t + AHEAD * THREADS; i < all; i += THREADS) load(i, *reinterpret_cast<uint4(*)[VECS]>(&rows[i]));
  }
  __syncthreads();
  auto finish = [&](int i, uint4 (&w)[VECS]) {
    const int k = tokens == 1 ? 0 : i / units, r = i - k * units, h = r / UNITS, u = r % UNITS;
    const Row to = row_of(a, tok0 + k, head_from + h, place[k][1], HEAD_BYTES);
    if (place[k][0] < 0 || to.dst == nullptr) return;   // a token that takes no part, a row without a slot
    if constexpr (FORM == HALF) {
      if (to.turn && u < turned) {
        float x[N], y[N];
        unpack<T>(w[0], x);
        unpack<T>(w[1], y);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 c = cs[k][u * N + e];
          const float p = x[e] * c.x - y[e] * c.y, q = x[e] * c.y + y[e] * c.x;
          x[e] = p;
          y[e] = q;
        }
        w[0] = packed<T>(x);
        w[1] = packed<T>(y);
      }
      __stcs(reinterpret_cast<uint4*>(to.dst) + (u < turned ? u : 2 * u), w[0]);
      __stcs(reinterpret_cast<uint4*>(to.dst) + (u < turned ? u + turned : 2 * u + 1), w[1]);
    } else if constexpr (FORM == INTERLEAVED) {
      if (to.turn && u * N < a.rot) {
        float x[N];
        unpack<T>(w[0], x);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          if (u * N + e < a.rot) {
            const float2 c = cs[k][(u * N + e) / 2];
            const float p = x[e] * c.x - x[e + 1] * c.y, q = x[e] * c.y + x[e + 1] * c.x;
            x[e] = p;
            x[e + 1] = q;
          }
        }
        w[0] = packed<T>(x);
      }
      __stcs(reinterpret_cast<uint4*>(to.dst) + u, w[0]);
    } else {
      w[0] = rows[i];
      if (to.turn && u * N < a.rot) {
        const T* row = reinterpret_cast<const T*>(rows + i - u);
        float x[N];
        unpack<T>(w[0], x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int at = u * N + e;
          if (at < half) {
            const float2 c = cs[k][at];
            x[e] = x[e] * c.x - (float)row[at + half] * c.y;
          } else if (at < a.rot) {
            const float2 c = cs[k][at - half];
            x[e] = (float)row[at - half] * c.y + x[e] * c.x;
          }
        }
        w[0] = packed<T>(x);
      }
      __stcs(reinterpret_cast<uint4*>(to.dst) + u, w[0]);
    }
  };
#pragma unroll
  for (int n = 0; n < AHEAD; ++n)
    if (t + n * THREADS < all) finish(t + n * THREADS, ahead[n]);
#pragma unroll 2
  for (int i = t + AHEAD * THREADS; i < all; i += THREADS) {
    uint4 w[VECS];
    if (FORM != STAGED) load(i, w);
    finish(i, w);
  }
}

template <typename T, int D, int FORM>
cudaError_t launch_form(const RopeArgs& a, int heads, int head_from, cudaStream_t st) {
  // Up to 64 heads of a token (STAGED keeps the rows in shared memory: 32 KB at most), and so many tokens as make 512 units, as
  // long as there are eight blocks for every SM all the same (8191 appended 38 us with one token a block, 31 so).  Where there are,
  // blocks of 128 threads, more of which fit an SM at different stages (65536 tokens 239 us with 256, 233 with 128; 8191 appended 30
  // and 26); else 256, which are through sooner (64 tokens 2.5 and 2.9).
  constexpr int UNITS = FORM == HALF ? D / (2 * Vec<T>::N) : D / Vec<T>::N;
  const int per_block = std::min(heads, 64);
  int tokens = std::max(1, std::min(MAX_TOKENS, 512 / (per_block * UNITS)));
  while (tokens > 1 && a.n_tokens / tokens < 8 * sm_count()) tokens /= 2;
  const int bytes = FORM == STAGED ? tokens * per_block * D * (int)sizeof(T) : 0;
  const dim3 grid((a.n_tokens + tokens - 1) / tokens, (heads + per_block - 1) / per_block);
  const cudaError_t e = grid.x * (int64_t)grid.y >= 8 * sm_count()
      ? launch_pdl(rope_kernel<T, D, FORM, 128>, grid, dim3(128), bytes, st, a, heads, head_from, per_block, tokens)
      : launch_pdl(rope_kernel<T, D, FORM, 256>, grid, dim3(256), bytes, st, a, heads, head_from, per_block, tokens);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_type(const RopeArgs& a, cudaStream_t st) {
  const int head_from = a.q != nullptr ? 0 : a.Hq;
  const int heads = (a.q != nullptr ? a.Hq : 0) + (a.k != nullptr ? a.Hkv : 0) + (a.v != nullptr ? a.Hkv : 0);
  if (a.interleaved) return launch_form<T, D, INTERLEAVED>(a, heads, head_from, st);
  if (a.rot / 2 % Vec<T>::N == 0) return launch_form<T, D, HALF>(a, heads, head_from, st);
  return launch_form<T, D, STAGED>(a, heads, head_from, st);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  if (a.dtype == EARN_F32) return a.D == 64 ? launch_type<float, 64>(a, st) : launch_type<float, 128>(a, st);
  return a.D == 64 ? launch_type<__nv_bfloat16, 64>(a, st) : launch_type<__nv_bfloat16, 128>(a, st);
}

}  // namespace earn

// Rotary positions: pairs of a head's first `rot` elements are turned by angle f_i * position and scaled by the amplitude,
//   y_a = A (x_a cos - x_b sin),  y_b = A (x_a sin + x_b cos),   pair i = (i, i + rot/2), or (2i, 2i + 1) interleaved;
// the rest of the head is copied.  The gradient is the transposed turn (sin negated).  In the append form the rows of K go,
// turned, and those of V, as they are, to their slots in the page pool.
//
// Bound by HBM: every row is read and written once.  Angles cost a token rot/2 sines and cosines, shared by all its heads:
// the product position * f_i is taken and reduced to turns in 64 bits (a 32-bit product is off by 0.06 rad at position 10^6),
// the remainder's sine and cosine in 32.  They go to shared memory, from where the threads take them, eight pairs at a time.
#include <algorithm>

#include "chunk_step.cuh"

namespace earn {
namespace {

constexpr int THREADS = 256;

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

template <typename T, int D, int FORM, int TOKENS>
__global__ void __launch_bounds__(THREADS) rope_kernel(RopeArgs a, int heads, int head_from, int per_block) {
  constexpr int N = Vec<T>::N, HEAD_BYTES = D * (int)sizeof(T);
  constexpr int UNITS = FORM == HALF ? D / (2 * N) : D / N;   // HALF: a unit is two vectors, a pair's halves or two that are copied
  __shared__ float2 cs[TOKENS][D / 2];
  __shared__ int place[TOKENS][2];   // position, slot
  extern __shared__ uint4 rows[];    // STAGED: the rows of the token
  const int t = threadIdx.x, tok0 = blockIdx.x * TOKENS, half = a.rot / 2;
  head_from += (int)blockIdx.y * per_block;   // this block's heads
  heads = min(per_block, heads - (int)blockIdx.y * per_block);
  pdl_launch_dependents();
  pdl_wait();
  if (t < TOKENS) {
    place[t][0] = tok0 + t < a.n_tokens ? a.positions[tok0 + t] : -1;
    place[t][1] = tok0 + t < a.n_tokens && a.slots != nullptr ? a.slots[tok0 + t] : -1;
  }
  for (int i = t; i < TOKENS * half; i += THREADS) {
    const int k = i / half, p = i - k * half;
    const int pos = tok0 + k < a.n_tokens ? a.positions[tok0 + k] : -1;
    const double turns = (double)pos * a.freq[p] * 0.15915494309189533577;   // 1 / (2 pi)
    float sn, cn;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cn);
    cs[k][p] = make_float2(a.amplitude * cn, a.sign * a.amplitude * sn);
  }
  __syncthreads();
  const int all = heads * UNITS;
#pragma unroll 1
  for (int k = 0; k < TOKENS; ++k) {
    if (place[k][0] < 0) continue;   // a token that takes no part (the whole block skips it)
    const int tok = tok0 + k, slot = place[k][1];
    if constexpr (FORM == STAGED) {
      for (int i = t; i < all; i += THREADS) rows[i] = reinterpret_cast<const uint4*>(row_of(a, tok, head_from + i / UNITS, slot, HEAD_BYTES).src)[i % UNITS];
      __syncthreads();
    }
#pragma unroll 2
    for (int i = t; i < all; i += THREADS) {
      const int h = i / UNITS, u = i % UNITS;
      const Row r = row_of(a, tok, head_from + h, slot, HEAD_BYTES);
      if (r.dst == nullptr) continue;
      if constexpr (FORM == HALF) {
        // pairs' units first: vectors u and u + half / N; then the copied ones, two by two behind the turned share
        const int turned = half / N, va = u < turned ? u : 2 * u, vb = u < turned ? u + turned : 2 * u + 1;
        uint4 wa = reinterpret_cast<const uint4*>(r.src)[va], wb = reinterpret_cast<const uint4*>(r.src)[vb];
        if (r.turn && u < turned) {
          float x[N], y[N];
          unpack<T>(wa, x);
          unpack<T>(wb, y);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 c = cs[k][u * N + e];
            const float p = x[e] * c.x - y[e] * c.y, q = x[e] * c.y + y[e] * c.x;
            x[e] = p;
            y[e] = q;
          }
          wa = packed<T>(x);
          wb = packed<T>(y);
        }
        reinterpret_cast<uint4*>(r.dst)[va] = wa;
        reinterpret_cast<uint4*>(r.dst)[vb] = wb;
      } else if constexpr (FORM == INTERLEAVED) {
        uint4 w = reinterpret_cast<const uint4*>(r.src)[u];
        if (r.turn && u * N < a.rot) {
          float x[N];
          unpack<T>(w, x);
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            if (u * N + e < a.rot) {
              const float2 c = cs[k][(u * N + e) / 2];
              const float p = x[e] * c.x - x[e + 1] * c.y, q = x[e] * c.y + x[e + 1] * c.x;
              x[e] = p;
              x[e + 1] = q;
            }
          }
          w = packed<T>(x);
        }
        reinterpret_cast<uint4*>(r.dst)[u] = w;
      } else {
        uint4 w = rows[i];
        if (r.turn && u * N < a.rot) {
          const T* row = reinterpret_cast<const T*>(rows + h * UNITS);
          float x[N];
          unpack<T>(w, x);
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
          w = packed<T>(x);
        }
        reinterpret_cast<uint4*>(r.dst)[u] = w;
      }
    }
    if constexpr (FORM == STAGED) __syncthreads();
  }
}

template <typename T, int D, int FORM, int TOKENS>
cudaError_t launch_form(const RopeArgs& a, int heads, int head_from, cudaStream_t st) {
  // a block takes up to 64 heads of a token (STAGED keeps their rows in shared memory: 32 KB at most)
  const int per_block = std::min(heads, 64);
  const int bytes = FORM == STAGED ? per_block * D * (int)sizeof(T) : 0;
  const dim3 grid((a.n_tokens + TOKENS - 1) / TOKENS, (heads + per_block - 1) / per_block);
  const cudaError_t e = launch_pdl(rope_kernel<T, D, FORM, TOKENS>, grid, dim3(THREADS), bytes, st, a, heads, head_from, per_block);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_type(const RopeArgs& a, cudaStream_t st) {
  const int head_from = a.q != nullptr ? 0 : a.Hq;
  const int heads = (a.q != nullptr ? a.Hq : 0) + (a.k != nullptr ? a.Hkv : 0) + (a.v != nullptr ? a.Hkv : 0);
  if (a.interleaved) return launch_form<T, D, INTERLEAVED, 1>(a, heads, head_from, st);
  if (a.rot / 2 % Vec<T>::N == 0) return launch_form<T, D, HALF, 1>(a, heads, head_from, st);
  return launch_form<T, D, STAGED, 1>(a, heads, head_from, st);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  if (a.dtype == EARN_F32) return a.D == 64 ? launch_type<float, 64>(a, st) : launch_type<float, 128>(a, st);
  return a.D == 64 ? launch_type<__nv_bfloat16, 64>(a, st) : launch_type<__nv_bfloat16, 128>(a, st);
}

}  // namespace earn

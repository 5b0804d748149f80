// Accumulated attention weight of the prompt's rows (earn_key_weights) on the CUDA cores: fp32 tensors, and bf16 shapes
// the tensor-core kernel does not take.  A CTA owns 128 keys of one (sequence, kv head) -- 32 where that leaves the grid
// small -- and walks the (query row, head of the group) pairs of the sequence's window in tiles of 64 columns; the logits are
// register-blocked 8 x 4 (2 x 4) over 256 threads.  Every weight is summed by
// one CTA in one order.  FMA-bound, with three 16-byte shared-memory reads per 32 products (23 TFLOP/s, 8 whole prompts of 1024 rows at 32/8 heads: 1.47 ms).
#include "paged_cache.cuh"

namespace earn {
namespace {

constexpr int TQ = 64;

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&x)[4]) { Elem<T>::load4(p, x); }

// Columns of D that are in shared memory at a time: a few where the grid is large and two CTAs are to share an SM, all of them
// where the call is a chain of latencies.
template <int D, int TK>
__host__ __device__ constexpr int q_depth() { return TK >= 128 ? 32 : D; }

// TK keys per CTA (a multiple of 32): thread (ty, tx) of 16 x 16 holds keys ty * KM .. and columns tx * 4 ..
template <typename T, int D, int TK>
__global__ void __launch_bounds__(256) key_weights_simt_kernel(KeyWeightArgs a) {
  constexpr int KM = TK / 16, KP = TK + 4, QP = TQ + 4;   // pitches of the transposed tiles
  constexpr int TD = q_depth<D, TK>();
  extern __shared__ __align__(16) float dyn[];
  float* ks = dyn;              // [D][KP]: all of the keys' columns, loaded once
  float* qs = dyn + D * KP;     // [TD][QP]
  __shared__ float lse[TQ];
  __shared__ int row_of[TQ];    // query row (position in the sequence) of a column, -1: none
  __shared__ int64_t q_at[TQ];  // element offset of its query
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int key0 = blockIdx.x * TK, kvh = blockIdx.y, b = blockIdx.z, g = a.Hq / a.Hkv;
  const int lo = a.cu_seqlens[b], len = min(a.cu_seqlens[b + 1] - lo, a.max_seqlen);
  if (key0 >= len) return;
  const T *q = reinterpret_cast<const T*>(a.q), *k = reinterpret_cast<const T*>(a.k);
  // four columns of a key at a time; neighbouring lanes take neighbouring keys so that the transposed stores do not collide
#pragma unroll 4
  for (int i = tid; i < TK * (D / 4); i += 256) {
    const int r = i % TK, d = i / TK * 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (key0 + r < len) load4(k + ((int64_t)(lo + key0 + r) * a.Hkv + kvh) * D + d, x);
#pragma unroll
    for (int c = 0; c < 4; ++c) ks[(d + c) * KP + r] = x[c];
  }
  const int first = max(len - a.n_obs > 0 ? len - a.n_obs : 0, key0);   // rows in front of key0 see none of these keys
  const int64_t n_cols = (int64_t)(len - first) * g;
  // A thread's terms of a tile are summed by themselves, tiles in sixteens, and those into the key's sum: a chain over all
  // of a long window's terms rounds each of them at the size of the whole sum (8192 rows, groups of 8: 4096 terms a thread).
  // (Selects at the end of the loop: with a branch for the sixteenth tile the small form's loop takes a sixth longer.)
  float sum[KM], sum16[KM];
#pragma unroll
  for (int i = 0; i < KM; ++i) sum[i] = sum16[i] = 0.f;
  int tile = 0;
  for (int64_t c0 = 0; c0 < n_cols; c0 += TQ) {
    __syncthreads();   // the last tile's columns have been used
    if (tid < TQ) {
      const bool in = c0 + tid < n_cols;
      const int row = in ? first + (int)((c0 + tid) / g) : -1, h = kvh * g + (int)((c0 + tid) % g);
      row_of[tid] = row;
      q_at[tid] = in ? ((int64_t)(lo + row) * a.Hq + h) * D : -1;
      lse[tid] = in ? a.lse[(int64_t)h * a.total + lo + row] : 0.f;
    }
    float s[KM][4] = {};
    for (int d0 = 0; d0 < D; d0 += TD) {
      __syncthreads();
#pragma unroll
      for (int i = tid; i < TQ * (TD / 4); i += 256) {
        const int c = i % TQ, d = i / TQ * 4;
        const int64_t at = q_at[c];
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (at >= 0) load4(q + at + d0 + d, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) qs[(d + e) * QP + c] = x[e];
      }
      __syncthreads();
#pragma unroll 8
      for (int d = 0; d < TD; ++d) {
        const float4 qq = *reinterpret_cast<const float4*>(qs + d * QP + tx * 4);
        const float qv[4] = {qq.x, qq.y, qq.z, qq.w};
        float kv[KM];
        if constexpr (KM % 4 == 0) {
#pragma unroll
          for (int i = 0; i < KM; i += 4) *reinterpret_cast<float4*>(kv + i) = *reinterpret_cast<const float4*>(ks + (d0 + d) * KP + ty * KM + i);
        } else {
          *reinterpret_cast<float2*>(kv) = *reinterpret_cast<const float2*>(ks + (d0 + d) * KP + ty * KM);
        }
#pragma unroll
        for (int i = 0; i < KM; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] = fmaf(kv[i], qv[j], s[i][j]);
      }
    }
    float sum1[KM];
#pragma unroll
    for (int i = 0; i < KM; ++i) sum1[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row_of[tx * 4 + j];
      const float d = lse[tx * 4 + j];
#pragma unroll
      for (int i = 0; i < KM; ++i)
        if (row >= key0 + ty * KM + i) sum1[i] += exp2f(fmaf(s[i][j], a.scale, -d) * kLog2e);   // causal; columns that do not exist: row -1
    }
#pragma unroll
    for (int i = 0; i < KM; ++i) sum16[i] += sum1[i];
    const bool full = (++tile & 15) == 0;
#pragma unroll
    for (int i = 0; i < KM; ++i) {
      sum[i] += full ? sum16[i] : 0.f;
      sum16[i] = full ? 0.f : sum16[i];
    }
  }
#pragma unroll
  for (int i = 0; i < KM; ++i) {
    sum[i] += sum16[i];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if (tx == 0 && key0 + ty * KM + i < len) a.weight[(int64_t)kvh * a.total + lo + key0 + ty * KM + i] = sum[i];
  }
}

template <typename T, int D, int TK>
cudaError_t launch_tk(const KeyWeightArgs& a, cudaStream_t st) {
  constexpr int smem = (D * (TK + 4) + q_depth<D, TK>() * (TQ + 4)) * 4;
  cudaError_t e = ensure_dynamic_smem<key_weights_simt_kernel<T, D, TK>>(smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(key_weights_simt_kernel<T, D, TK>, dim3((a.max_seqlen + TK - 1) / TK, a.Hkv, a.batch), dim3(256), smem, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_t(const KeyWeightArgs& a, cudaStream_t st) {
  const int64_t big = (int64_t)((a.max_seqlen + 127) / 128) * a.Hkv * a.batch;
  return big >= 2 * sm_count() ? launch_tk<T, D, 128>(a, st) : launch_tk<T, D, 32>(a, st);
}

}  // namespace

cudaError_t launch_key_weights_simt(const KeyWeightArgs& a, cudaStream_t st) {
  if (a.dtype == EARN_F32) return a.D == 64 ? launch_t<float, 64>(a, st) : launch_t<float, 128>(a, st);
  return a.D == 64 ? launch_t<__nv_bfloat16, 64>(a, st) : launch_t<__nv_bfloat16, 128>(a, st);
}

}  // namespace earn

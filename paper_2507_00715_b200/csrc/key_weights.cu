// Accumulated attention weight of the prompt's rows (earn_key_weights) on the CUDA cores: fp32 tensors, and bf16 shapes
// the tensor-core kernel does not take.  A CTA owns 64 keys of one (sequence, kv head) and walks the (query row, head of
// the group) pairs of the sequence's window in tiles of 64; the 64 x 64 logits are register-blocked 4 x 4 over 256 threads.
// Every weight is summed by one CTA in one order.  FMA-bound: 2 D flops per pair from 64-row tiles in shared memory.
#include "earn_common.cuh"

namespace earn {
namespace {

constexpr int TK = 64, TQ = 64, PITCH = TK + 4;   // floats per column of the transposed tiles

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T, int D>
__global__ void __launch_bounds__(256) key_weights_simt_kernel(KeyWeightArgs a) {
  extern __shared__ __align__(16) float tiles[];
  float* ks = tiles;               // [D][PITCH]
  float* qs = tiles + D * PITCH;   // [D][PITCH]
  __shared__ float lse2[TQ];
  __shared__ int row_of[TQ];       // query row (position in the sequence) of a column, -1: none
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int key0 = blockIdx.x * TK, kvh = blockIdx.y, b = blockIdx.z, g = a.Hq / a.Hkv;
  const int lo = a.cu_seqlens[b], len = min(a.cu_seqlens[b + 1] - lo, a.max_seqlen);
  if (key0 >= len) return;
  const T *q = reinterpret_cast<const T*>(a.q), *k = reinterpret_cast<const T*>(a.k);
  for (int i = tid; i < TK * D; i += 256) {
    const int r = i / D, d = i % D;
    ks[d * PITCH + r] = key0 + r < len ? to_f(k[((int64_t)(lo + key0 + r) * a.Hkv + kvh) * D + d]) : 0.f;
  }
  const float scale_log2 = a.scale * kLog2e;
  const int first = max(len - a.n_obs > 0 ? len - a.n_obs : 0, key0);   // rows in front of key0 see none of these keys
  const int64_t n_cols = (int64_t)(len - first) * g;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t c0 = 0; c0 < n_cols; c0 += TQ) {
    __syncthreads();   // the last tile has been read
    if (tid < TQ) {
      const bool in = c0 + tid < n_cols;
      const int row = in ? first + (int)((c0 + tid) / g) : -1, h = kvh * g + (int)((c0 + tid) % g);
      row_of[tid] = row;
      lse2[tid] = in ? a.lse[(int64_t)h * a.total + lo + row] * kLog2e : 0.f;
    }
    for (int i = tid; i < TQ * D; i += 256) {
      const int c = i / D, d = i % D;
      const int64_t at = c0 + c;
      qs[d * PITCH + c] = at < n_cols ? to_f(q[((int64_t)(lo + first + at / g) * a.Hq + kvh * g + at % g) * D + d]) : 0.f;
    }
    __syncthreads();
    float s[4][4] = {};
#pragma unroll 4
    for (int d = 0; d < D; ++d) {
      const float4 kk = *reinterpret_cast<const float4*>(ks + d * PITCH + ty * 4);
      const float4 qq = *reinterpret_cast<const float4*>(qs + d * PITCH + tx * 4);
      const float kv[4] = {kk.x, kk.y, kk.z, kk.w}, qv[4] = {qq.x, qq.y, qq.z, qq.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = fmaf(kv[i], qv[j], s[i][j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row_of[tx * 4 + j];
      const float d = lse2[tx * 4 + j];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row >= key0 + ty * 4 + i) sum[i] += exp2f(fmaf(s[i][j], scale_log2, -d));   // causal; columns that do not exist: row -1
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if (tx == 0 && key0 + ty * 4 + i < len) a.weight[(int64_t)kvh * a.total + lo + key0 + ty * 4 + i] = sum[i];
  }
}

template <typename T, int D>
cudaError_t launch_t(const KeyWeightArgs& a, cudaStream_t st) {
  constexpr int smem = 2 * D * PITCH * 4;
  cudaError_t e = ensure_dynamic_smem<key_weights_simt_kernel<T, D>>(smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(key_weights_simt_kernel<T, D>, dim3((a.max_seqlen + TK - 1) / TK, a.Hkv, a.batch), dim3(256), smem, st, a);
  note_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_key_weights_simt(const KeyWeightArgs& a, cudaStream_t st) {
  if (a.dtype == EARN_F32) return a.D == 64 ? launch_t<float, 64>(a, st) : launch_t<float, 128>(a, st);
  return a.D == 64 ? launch_t<__nv_bfloat16, 64>(a, st) : launch_t<__nv_bfloat16, 128>(a, st);
}

}  // namespace earn

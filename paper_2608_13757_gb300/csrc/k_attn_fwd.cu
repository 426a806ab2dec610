// Forward attention over packed sequences, one warp per query row and head.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn.h"

namespace syncgb {
namespace {

__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(__nv_bfloat16& y, float x) { y = __float2bfloat16(x); }
__device__ __forceinline__ void from_f(__half& y, float x) { y = __float2half(x); }

template <class T>
__device__ __forceinline__ const T* at(const AttnTensor& t, int64_t row, int head) {
  return static_cast<const T*>(t.data) + row * t.row + head * t.head;
}

__device__ __forceinline__ float sum_warp(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

template <class T>
__device__ __forceinline__ void load_row(const T* p, int dim, int lane, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = lane + 32 * i < dim ? to_f(p[lane + 32 * i]) : 0.f;
}

template <class T>
__global__ void __launch_bounds__(256) k_attn_rows(const __grid_constant__ AttnArgs a) {
  const AttnItem it = a.q_item[blockIdx.x];
  const AttnSeq s = a.seq[it.seq];
  const int lane = threadIdx.x % 32, kh = it.head / (a.heads / a.kv_heads);
  for (int r = it.tile * kTile + threadIdx.x / 32; r < min(s.lq, (it.tile + 1) * kTile); r += 8) {
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    load_row(at<T>(a.q, s.q0 + r, it.head), a.dim, lane, q);
    for (int j = 0; j <= r + s.lk - s.lq; ++j) {
      float k[4], v[4];
      load_row(at<T>(a.k, s.k0 + j, kh), a.dim, lane, k);
      load_row(at<T>(a.v, s.k0 + j, kh), a.dim, lane, v);
      const float e = sum_warp(q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3]) * a.scale;
      const float n = fmaxf(m, e), w = n == -INFINITY ? 1.f : expf(m - n), p = n == -INFINITY ? 0.f : expf(e - n);
      l = l * w + p;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = o[i] * w + p * v[i];
      m = n;
    }
    T* out = static_cast<T*>(a.o.data) + (s.q0 + r) * a.o.row + it.head * a.o.head;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 32 * i < a.dim) from_f(out[lane + 32 * i], l > 0.f ? o[i] / l : l == 0.f ? 0.f : o[i] + l);
    if (a.lse && lane == 0) a.lse[it.head * a.q.rows + s.q0 + r] = l == 0.f ? -INFINITY : m + logf(l);
  }
}

}  // namespace

cudaError_t launch_attn_forward(const AttnArgs& a, cudaStream_t st) {
  if (a.bf16)
    k_attn_rows<__nv_bfloat16><<<a.n_q_items, 256, 0, st>>>(a);
  else
    k_attn_rows<__half><<<a.n_q_items, 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace syncgb

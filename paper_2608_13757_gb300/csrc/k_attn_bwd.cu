// Gradients of attention over packed sequences: one warp per query row for
// dq, one per key row for dk and dv (summed over the query heads of its key
// head), so that nothing is added out of order.
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
__device__ __forceinline__ T* at(const AttnTensor& t, int64_t row, int head) {
  return static_cast<T*>(t.data) + row * t.row + head * t.head;
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
__device__ __forceinline__ void store_row(T* p, int dim, int lane, const float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < dim) from_f(p[lane + 32 * i], x[i]);
}
__device__ __forceinline__ float dot(const float* x, const float* y) {
  return sum_warp(x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3]);
}

template <class T>
__global__ void __launch_bounds__(256) k_attn_dq(const __grid_constant__ AttnArgs a) {
  const AttnTile it = a.q_tile[blockIdx.x];
  const AttnSeq s = a.seq[it.seq];
  const int lane = threadIdx.x % 32, kh = it.head / (a.heads / a.kv_heads);
  for (int r = it.tile * kTile + threadIdx.x / 32; r < min(s.lq, (it.tile + 1) * kTile); r += 8) {
    float q[4], o[4], g[4], dq[4] = {0.f, 0.f, 0.f, 0.f};
    load_row(at<T>(a.q, s.q0 + r, it.head), a.dim, lane, q);
    load_row(at<T>(a.o, s.q0 + r, it.head), a.dim, lane, o);
    load_row(at<T>(a.d_o, s.q0 + r, it.head), a.dim, lane, g);
    const float delta = dot(o, g), lse = a.lse[it.head * a.q.rows + s.q0 + r];
    if (lane == 0) a.delta[it.head * a.delta_rows + s.q0 + r] = delta;
    for (int j = 0; j <= r + s.lk - s.lq; ++j) {
      float k[4], v[4];
      load_row(at<T>(a.k, s.k0 + j, kh), a.dim, lane, k);
      load_row(at<T>(a.v, s.k0 + j, kh), a.dim, lane, v);
      const float p = lse == -INFINITY ? 0.f : expf(dot(q, k) * a.scale - lse);
      const float ds = p * (dot(g, v) - delta) * a.scale;
#pragma unroll
      for (int i = 0; i < 4; ++i) dq[i] += ds * k[i];
    }
    store_row(at<T>(a.dq, s.q0 + r, it.head), a.dim, lane, dq);
  }
}

template <class T>
__global__ void __launch_bounds__(256) k_attn_dkv(const __grid_constant__ AttnArgs a) {
  const AttnTile it = a.k_tile[blockIdx.x];
  const AttnSeq s = a.seq[it.seq];
  const int lane = threadIdx.x % 32, group = a.heads / a.kv_heads;
  for (int j = it.tile * kTile + threadIdx.x / 32; j < min(s.lk, (it.tile + 1) * kTile); j += 8) {
    float k[4], v[4], dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
    load_row(at<T>(a.k, s.k0 + j, it.head), a.dim, lane, k);
    load_row(at<T>(a.v, s.k0 + j, it.head), a.dim, lane, v);
    for (int h = it.head * group; h < (it.head + 1) * group; ++h)
      for (int r = max(0, j + s.lq - s.lk); r < s.lq; ++r) {
        float q[4], g[4];
        load_row(at<T>(a.q, s.q0 + r, h), a.dim, lane, q);
        load_row(at<T>(a.d_o, s.q0 + r, h), a.dim, lane, g);
        const float lse = a.lse[h * a.q.rows + s.q0 + r];
        const float p = lse == -INFINITY ? 0.f : expf(dot(q, k) * a.scale - lse);
        const float ds = p * (dot(g, v) - a.delta[h * a.delta_rows + s.q0 + r]) * a.scale;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dk[i] += ds * q[i];
          dv[i] += p * g[i];
        }
      }
    store_row(at<T>(a.dk, s.k0 + j, it.head), a.dim, lane, dk);
    store_row(at<T>(a.dv, s.k0 + j, it.head), a.dim, lane, dv);
  }
}

template <class T>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  if (a.n_q_tiles) {
    k_attn_dq<T><<<a.n_q_tiles, 256, 0, st>>>(a);
    if (cudaError_t e = cudaGetLastError()) return e;
    count_launch();
  }
  if (a.n_k_tiles) {
    k_attn_dkv<T><<<a.n_k_tiles, 256, 0, st>>>(a);
    if (cudaError_t e = cudaGetLastError()) return e;
    count_launch();
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_attn_backward(const AttnArgs& a, cudaStream_t st) {
  return a.bf16 ? launch<__nv_bfloat16>(a, st) : launch<__half>(a, st);
}

}  // namespace syncgb

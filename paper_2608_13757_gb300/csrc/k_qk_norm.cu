// Norm of every query and key head with the position rotation in the same
// pass, and its gradient (include/sync.h, sync_qk_norm_rope).
//
// One pass over the data, bound by memory: a head's entries are read once,
// held in registers through the norm's sum and the rotation, and written
// once.  A head is taken by LANES lanes with up to VEC pairs of entries each;
// both entries of a pair sit in one lane, so the rotation moves nothing
// between lanes.  Entries that are not rotated form pairs too, with c = 1 and
// s = 0.  A warp stays with one token for several heads and reads its angles
// once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "norm.h"
#include "sync.h"

namespace syncgb {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(__nv_bfloat16& y, float x) { y = __float2bfloat16(x); }
__device__ __forceinline__ void from_f(__half& y, float x) { y = __float2half(x); }

// N consecutive entries, in one access
template <class T, int N>
struct alignas(N * sizeof(T)) Pack {
  T x[N];
};
template <int N, class T>
__device__ __forceinline__ void load(const T* p, float* f) {
  const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = to_f(v.x[i]);
}
template <int N, class T>
__device__ __forceinline__ void store(T* p, const float* f) {
  Pack<T, N> v;
#pragma unroll
  for (int i = 0; i < N; ++i) from_f(v.x[i], f[i]);
  *reinterpret_cast<Pack<T, N>*>(p) = v;
}

// How a lane reads and writes its pairs: x[0..VEC) holds their first entries,
// x[VEC..2*VEC) their second ones.
//   VECTOR: VEC pairs that are all rotated or all not; two accesses of VEC
//     entries (the host has checked sizes and alignment);
//   otherwise entry by entry, each pair on its own, for sizes, strides and
//     addresses that no wide access fits.
template <class T, int VEC_, int LANES_, bool INTER, bool VECTOR>
struct Shape {
  static constexpr int VEC = VEC_, LANES = LANES_;
  int first, pairs, half, rest, rotated;
  __device__ __forceinline__ explicit Shape(const NormArgs& a)
      : first((int)(threadIdx.x % LANES) * VEC), pairs(a.dim / 2), half(a.rotated / 2),
        rest((a.dim - a.rotated) / 2), rotated(a.rotated) {}
  __device__ __forceinline__ bool on() const { return first < pairs; }
  __device__ __forceinline__ bool has(int i) const { return VECTOR ? on() : first + i < pairs; }
  __device__ __forceinline__ bool turns(int i) const { return first + (VECTOR ? 0 : i) < half; }
  // offsets of a pair's entries in the head
  __device__ __forceinline__ int lo(int i) const {
    const int p = first + i;
    return INTER ? 2 * p : p < half ? p : rotated + p - half;
  }
  __device__ __forceinline__ int hi(int i) const {
    return lo(i) + (INTER ? 1 : first + i < half ? half : rest);
  }
  template <class P>
  __device__ __forceinline__ void read(const P* p, float* x) const {
    if constexpr (VECTOR && INTER) {
      float y[2 * VEC];
      load<VEC>(p + lo(0), y);
      load<VEC>(p + lo(0) + VEC, y + VEC);
#pragma unroll
      for (int i = 0; i < VEC; ++i) { x[i] = y[2 * i]; x[VEC + i] = y[2 * i + 1]; }
    } else if constexpr (VECTOR) {
      load<VEC>(p + lo(0), x);
      load<VEC>(p + hi(0), x + VEC);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (has(i)) { x[i] = to_f(p[lo(i)]); x[VEC + i] = to_f(p[hi(i)]); }
    }
  }
  template <class P>
  __device__ __forceinline__ void write(P* p, const float* x) const {
    if constexpr (VECTOR && INTER) {
      float y[2 * VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) { y[2 * i] = x[i]; y[2 * i + 1] = x[VEC + i]; }
      store<VEC>(p + lo(0), y);
      store<VEC>(p + lo(0) + VEC, y + VEC);
    } else if constexpr (VECTOR) {
      store<VEC>(p + lo(0), x);
      store<VEC>(p + hi(0), x + VEC);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (has(i)) { from_f(p[lo(i)], x[i]); from_f(p[hi(i)], x[VEC + i]); }
    }
  }
  __device__ __forceinline__ void weights(const void* w, float* x) const {
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) x[i] = 1.f;
    if (w && on()) read(static_cast<const T*>(w), x);
  }
  // the angles of a token; NaN for a position outside the table
  __device__ __forceinline__ void angles(const NormArgs& a, int64_t t, float* c, float* s) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i) { c[i] = 1.f; s[i] = 0.f; }
    const int64_t pos = a.positions ? (int64_t)__ldg(a.positions + t) : t;
    if (pos < 0 || pos >= a.n_positions) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
      return;
    }
    const int64_t at = pos * half + first;
    if constexpr (VECTOR) {
      if (on() && turns(0)) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) { load<4>(a.cos + at + i, c + i); load<4>(a.sin + at + i, s + i); }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (has(i) && turns(i)) { c[i] = __ldg(a.cos + at + i); s[i] = __ldg(a.sin + at + i); }
    }
  }
};

template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// Head h of the query heads followed by the key heads, at token t.
template <class T>
__device__ __forceinline__ T* head_of(const NormTensor& q, const NormTensor& k, int heads, int64_t t, int h) {
  return h < heads ? static_cast<T*>(q.data) + t * q.row + h * q.head
                   : static_cast<T*>(k.data) + t * k.row + (h - heads) * k.head;
}

// a.split warps share a token, a.per heads each.
template <class T, class S>
__global__ void __launch_bounds__(kThreads) k_norm_rope(const __grid_constant__ NormArgs a) {
  constexpr int VEC = S::VEC, G = 32 / S::LANES;   // G heads of a warp at a time
  const int64_t warp = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  const int64_t t = warp / a.split;
  if (t >= a.rows) return;
  const int h0 = (int)(warp - t * a.split) * a.per, h1 = min(a.heads + a.kv_heads, h0 + a.per);
  const S l(a);
  float c[VEC], s[VEC], wq[2 * VEC], wk[2 * VEC];
  l.angles(a, t, c, s);
  l.weights(a.q_weight, wq);
  l.weights(a.k_weight, wk);
  const int group = (threadIdx.x % 32) / S::LANES;
#pragma unroll 2
  for (int hb = h0; hb < h1; hb += G) {   // the same trips for every lane: the sums take whole warps
    const int h = hb + group;
    const bool on = l.on() && h < h1;
    float x[2 * VEC];
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) x[i] = 0.f;
    if (on) l.read(head_of<const T>(a.q, a.k, a.heads, t, h), x);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) ss += x[i] * x[i];
    const float r = rsqrtf(sum_lanes<S::LANES>(ss) * a.inv_dim + a.eps);
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float u = x[i] * r * (h < a.heads ? wq[i] : wk[i]);
      const float v = x[VEC + i] * r * (h < a.heads ? wq[VEC + i] : wk[VEC + i]);
      x[i] = u * c[i] - v * s[i];
      x[VEC + i] = v * c[i] + u * s[i];
    }
    l.write(head_of<T>(a.q_out, a.k_out, a.heads, t, h), x);
  }
}

// Gradient, with xh = r x the normed head: dx = r (w dz - xh mean(w dz xh)),
// dw = sum of dz xh, dz the output's gradient turned back.  Warps take
// (token, part of its heads) in turn; the weights' sums stay in registers
// until the end, go through shared memory in warp order and leave as one row
// per block, so their order does not depend on the run.
template <class T, class S>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope_grad(const __grid_constant__ NormArgs a) {
  constexpr int VEC = S::VEC, G = 32 / S::LANES;
  extern __shared__ float part[];         // [kWarps][q, k][dim]
  const S l(a);
  const int group = (threadIdx.x % 32) / S::LANES;
  float wq[2 * VEC], wk[2 * VEC], gq[2 * VEC], gk[2 * VEC];
  l.weights(a.q_weight, wq);
  l.weights(a.k_weight, wk);
#pragma unroll
  for (int i = 0; i < 2 * VEC; ++i) gq[i] = gk[i] = 0.f;
  const int64_t all = a.rows * a.split;
  for (int64_t warp = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32; warp < all; warp += gridDim.x * (int64_t)kWarps) {
    const int64_t t = warp / a.split;
    const int h0 = (int)(warp - t * a.split) * a.per, h1 = min(a.heads + a.kv_heads, h0 + a.per);
    float c[VEC], s[VEC];
    l.angles(a, t, c, s);
#pragma unroll 2
    for (int hb = h0; hb < h1; hb += G) {
      const int h = hb + group;
      const bool on = l.on() && h < h1, isq = h < a.heads;
      float x[2 * VEC], d[2 * VEC];
#pragma unroll
      for (int i = 0; i < 2 * VEC; ++i) x[i] = d[i] = 0.f;
      if (on) {
        l.read(head_of<const T>(a.q, a.k, a.heads, t, h), x);
        l.read(head_of<const T>(a.q_out, a.k_out, a.heads, t, h), d);
      }
      float ss = 0.f, xd = 0.f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {     // back through the rotation
        const float u = d[i], v = d[VEC + i];
        d[i] = u * c[i] + v * s[i];
        d[VEC + i] = v * c[i] - u * s[i];
      }
#pragma unroll
      for (int i = 0; i < 2 * VEC; ++i) {
        ss += x[i] * x[i];
        xd += x[i] * d[i] * (isq ? wq[i] : wk[i]);
      }
      const float r = rsqrtf(sum_lanes<S::LANES>(ss) * a.inv_dim + a.eps);
      const float m = sum_lanes<S::LANES>(xd) * a.inv_dim * r * r;
      if (!on) continue;
#pragma unroll
      for (int i = 0; i < 2 * VEC; ++i) {
        const float g = d[i] * x[i] * r;
        gq[i] += isq ? g : 0.f;
        gk[i] += isq ? 0.f : g;
        d[i] = r * (d[i] * (isq ? wq[i] : wk[i]) - x[i] * m);
      }
      l.write(head_of<T>(a.dq, a.dk, a.heads, t, h), d);
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * VEC; ++i)
#pragma unroll
    for (int o = S::LANES; o < 32; o <<= 1) {
      gq[i] += __shfl_xor_sync(~0u, gq[i], o);
      gk[i] += __shfl_xor_sync(~0u, gk[i], o);
    }
  if (group == 0) {
    float* row = part + threadIdx.x / 32 * 2 * a.dim;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (l.has(i)) {
        row[l.lo(i)] = gq[i];
        row[l.hi(i)] = gq[VEC + i];
        row[a.dim + l.lo(i)] = gk[i];
        row[a.dim + l.hi(i)] = gk[VEC + i];
      }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * a.dim; e += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += part[w * 2 * a.dim + e];
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + e] = v;
  }
}

// The blocks' rows summed in a fixed order: a block takes 32 columns, its
// warps take rows in turn, and the warps' sums are added in warp order.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_weights(const __grid_constant__ NormArgs a, int blocks) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, e = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (e < 2 * a.dim)
    for (int b = w; b < blocks; b += 32) v += a.partial[(int64_t)b * 2 * a.dim + e];
  part[w][lane] = v;
  __syncthreads();
  if (w || e >= 2 * a.dim) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) v += part[i][lane];
  T* out = static_cast<T*>(e < a.dim ? a.q_weight_grad : a.k_weight_grad);
  if (out) from_f(out[e < a.dim ? e : e - a.dim], v);
}

template <class T, class S>
cudaError_t launch(NormArgs a, cudaStream_t st) {
  // A token's heads go to as many warps as it takes to fill the GPU (32 warps
  // per SM are resident, about), in whole rounds of G heads.
  constexpr int G = 32 / S::LANES;
  const int rounds = (a.heads + a.kv_heads + G - 1) / G;
  const int64_t want = (int64_t)a.num_sms * 32;
  const int split = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, want / std::max<int64_t>(1, a.rows)));
  a.per = (rounds + split - 1) / split * G;
  a.split = (a.heads + a.kv_heads + a.per - 1) / a.per;
  const int64_t blocks = (a.rows * a.split + kWarps - 1) / kWarps;
  if (!a.grad) {
    if (blocks == 0) return cudaSuccess;
    k_norm_rope<T, S><<<(unsigned)blocks, kThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
  }
  const int n = (int)std::min<int64_t>(std::max<int64_t>(1, blocks), norm_blocks(a.num_sms));
  k_norm_rope_grad<T, S><<<n, kThreads, kWarps * 2 * a.dim * sizeof(float), st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  count_launch();
  if (!a.q_weight_grad && !a.k_weight_grad) return cudaSuccess;
  k_norm_weights<T><<<(2 * a.dim + 31) / 32, 1024, 0, st>>>(a, n);
  e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

// Whether accesses of V entries (and of 4 angles) fit all sizes, strides and addresses.
bool fits(const NormArgs& a, int V) {
  const int size = a.dtype == SYNC_FP32 ? 4 : 2;
  if (a.rotated / 2 % V || a.dim / 2 % V) return false;
  auto aligned = [](const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  auto ok = [&](const NormTensor& t) { return aligned(t.data, V * size) && t.row % V == 0 && t.head % V == 0; };
  if (!ok(a.q) || !ok(a.k) || !ok(a.q_out) || !ok(a.k_out) || (a.grad && (!ok(a.dq) || !ok(a.dk)))) return false;
  return aligned(a.q_weight, V * size) && aligned(a.k_weight, V * size) && aligned(a.cos, 16) && aligned(a.sin, 16);
}

template <class T, bool INTER>
cudaError_t pick(const NormArgs& a, cudaStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (fits(a, 8)) {
      if (a.dim <= 64) return launch<T, Shape<T, 8, 4, INTER, true>>(a, st);
      if (a.dim <= 128) return launch<T, Shape<T, 8, 8, INTER, true>>(a, st);
      return launch<T, Shape<T, 8, 16, INTER, true>>(a, st);
    }
    if (fits(a, 4) && a.dim <= 128) return launch<T, Shape<T, 4, 16, INTER, true>>(a, st);
  } else if (fits(a, 4)) {
    if (a.dim <= 64) return launch<T, Shape<T, 4, 8, INTER, true>>(a, st);
    if (a.dim <= 128) return launch<T, Shape<T, 4, 16, INTER, true>>(a, st);
    return launch<T, Shape<T, 4, 32, INTER, true>>(a, st);
  }
  return launch<T, Shape<T, 4, 32, INTER, false>>(a, st);
}

template <class T>
cudaError_t pick(const NormArgs& a, cudaStream_t st) {
  return a.interleaved ? pick<T, true>(a, st) : pick<T, false>(a, st);
}

}  // namespace

cudaError_t launch_norm_rope(const NormArgs& a, cudaStream_t st) {
  switch (a.dtype) {
    case SYNC_BF16: return pick<__nv_bfloat16>(a, st);
    case SYNC_FP16: return pick<__half>(a, st);
    default: return pick<float>(a, st);
  }
}

}  // namespace syncgb

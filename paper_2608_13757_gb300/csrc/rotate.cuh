// Heads turned by the angles of their token's positions: device code of the
// kernels that rotate.
//
// A block stages the angles of a few tokens in shared memory, pair by pair from
// the table rows of the pair's axis, and its threads then take runs of pairs of
// all heads in turn.  The products and their sum are rounded one by one (no
// fused multiply-add), so that a rotation has the same 32-bit value wherever it
// is computed; every use here is bound by memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cache.h"

namespace syncgb {
namespace rotate {

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(__nv_bfloat16& y, float x) { y = __float2bfloat16(x); }
__device__ __forceinline__ void from_f(__half& y, float x) { y = __float2half(x); }

// N consecutive entries, in one access of up to 16 bytes
template <class T, int N>
struct alignas(N * sizeof(T)) Pack {
  T x[N];
};

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
}

// The position of a row on the axis of pair j; `at` where none are given.
__device__ __forceinline__ int64_t position(const Rotation& r, int64_t row, int64_t at, int j) {
  if (!r.positions) return at;
  const int axis = r.axis[j / 16] >> (2 * (j % 16)) & 3;
  return __ldg(r.positions + axis * r.position_stride + row);
}
// The angle of pair j; NaN for a position outside the table.
__device__ __forceinline__ float2 angle(const Rotation& r, int64_t pos, int j) {
  if (pos < 0 || pos >= r.n_positions) return make_float2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
  const int64_t i = pos * r.half + j;
  return make_float2(__ldg(r.cos + i), r.way * __ldg(r.sin + i));
}

// A run of VEC pairs of a head from pair p on: where its first and second
// entries are.  Pairs from `half` on are the entries that are not turned.
template <class T, int VEC, bool INTER>
struct Pairs {
  static constexpr int kVec = VEC;
  alignas(VEC * sizeof(T)) T x[2 * VEC];   // as they were read: first entries, then second ones; INTER: in order
  static __device__ __forceinline__ int lo(int p, int half) { return INTER ? 2 * p : p < half ? p : half + p; }
  static __device__ __forceinline__ int hi(int p, int half, int pairs) { return INTER ? 2 * p + VEC : p < half ? half + p : pairs + p; }
  __device__ __forceinline__ void read(const T* head, int p, int half, int pairs) {
    *reinterpret_cast<Pack<T, VEC>*>(x) = *reinterpret_cast<const Pack<T, VEC>*>(head + lo(p, half));
    *reinterpret_cast<Pack<T, VEC>*>(x + VEC) = *reinterpret_cast<const Pack<T, VEC>*>(head + hi(p, half, pairs));
  }
  __device__ __forceinline__ void write(T* head, int p, int half, int pairs) const {
    *reinterpret_cast<Pack<T, VEC>*>(head + lo(p, half)) = *reinterpret_cast<const Pack<T, VEC>*>(x);
    *reinterpret_cast<Pack<T, VEC>*>(head + hi(p, half, pairs)) = *reinterpret_cast<const Pack<T, VEC>*>(x + VEC);
  }
  // by the angles of its pairs, cosines at c and sines at s
  __device__ __forceinline__ void by(const float* c, const float* s) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      T& u = x[INTER ? 2 * i : i];
      T& w = x[INTER ? 2 * i + 1 : VEC + i];
      float a = to_f(u), b = to_f(w);
      turn(a, b, c[i], s[i]);
      from_f(u, a);
      from_f(w, b);
    }
  }
};

// Items (token, head, run of a head) of a block in steps of its threads, counted
// on instead of divided out.
struct Walk {
  int t, h, r;
  int dt, dh, dr, heads, runs;
  __device__ __forceinline__ Walk(int from, int step, int heads_, int runs_) : heads(heads_), runs(runs_) {
    const int each = heads * runs;
    t = from / each;
    h = (from - t * each) / runs;
    r = from - t * each - h * runs;
    dt = step / each;
    dh = (step - dt * each) / runs;
    dr = step - dt * each - dh * runs;
  }
  __device__ __forceinline__ void next() {
    r += dr;
    h += dh;
    t += dt;
    if (r >= runs) {
      r -= runs;
      ++h;
    }
    if (h >= heads) {
      h -= heads;
      ++t;
    }
  }
};

// The widest run of pairs, of up to 16 bytes, that sizes, strides and
// addresses of all `n` tensors allow, in entries of `size` bytes; 1 always goes.
inline int widest(const HeadTensor* t, int n, int size, int half, int dim) {
  for (int vec = 16 / size; vec > 1; vec /= 2) {
    bool ok = vec * size >= 8 && half % vec == 0 && (dim / 2 - half) % vec == 0;
    for (int i = 0; i < n && ok; ++i)
      ok = reinterpret_cast<uintptr_t>(t[i].data) % (vec * size) == 0 && t[i].row % vec == 0 && t[i].head % vec == 0;
    if (ok) return vec;
  }
  return 1;
}

}  // namespace rotate
}  // namespace syncgb

// Heads turned by the angles of their token's positions: device code of the
// kernels that rotate, and how they go through their rows.
//
// A thread has a column, a run of entries of one head, for all the tokens that
// its block takes: `par` tokens side by side where a token has few columns, and
// `ahead` of them one after the other, whose reads are in flight together.  The
// angles of a group of tokens are staged in shared memory, pair by pair from the
// table rows of the pair's axis; blocks stay, and in k_rope a group's angles and
// positions are read while the one before it is turned.
//
// The products and their sum are rounded one by one (no fused multiply-add), so
// that a rotation has the same 32-bit value wherever it is computed; every use
// here is bound by memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "cache.h"

namespace syncgb {
namespace rotate {

// Threads of a block at most, and of an SM (which leaves a thread 96 registers);
// reads that a thread has in flight, and entries that it stages for a group.
constexpr int kMostThreads = 512, kResident = 640, kAhead = 4, kStaged = 2;

// How a kernel's blocks go through `rows` tokens of `columns` columns.
struct Columns {
  int each = 0;          // columns of a block: threads that one token takes
  int par = 1, ahead = 1, threads = 0;
  int batch = 1;         // groups whose angles are staged at a time (k_append)
  int blocks_x = 0, blocks_y = 0;
  int64_t groups = 0;
  __host__ __device__ int tokens() const { return par * ahead; }
};

// most_ahead: tokens that a thread may have in flight; stage: staged entries per
// token (0: none), of which a thread takes kStaged per group at most; most: columns
// of a block; resident: threads of an SM.
inline Columns columns_of(int64_t rows, int columns, int most_ahead, int stage, int num_sms, int most = kMostThreads, int resident = kResident) {
  Columns c;
  columns = (columns + 3) / 4 * 4;                          // four lanes share a group's scale
  c.blocks_y = (columns + most - 1) / most;
  c.each = c.blocks_y == 1 ? columns : ((columns + c.blocks_y - 1) / c.blocks_y + 31) / 32 * 32;
  c.par = std::max(1, 256 / c.each);
  // as long as every SM has a block, and the staging of a group stays small
  c.par = (int)std::max<int64_t>(1, std::min<int64_t>(c.par, rows / num_sms));
  c.threads = (std::max(c.par * c.each, (stage + kStaged - 1) / kStaged) + 31) / 32 * 32;
  while (c.par > 1 && c.par * stage > kStaged * c.threads) --c.par;
  c.ahead = most_ahead;
  const int64_t blocks = std::max<int64_t>(1, (int64_t)num_sms * std::max(1, resident / c.threads) / c.blocks_y);
  while (c.ahead > 1 && (c.tokens() * stage > kStaged * c.threads || rows < blocks * c.tokens())) c.ahead /= 2;
  c.groups = (rows + c.tokens() - 1) / c.tokens();
  c.blocks_x = (int)std::min<int64_t>(c.groups, blocks);
  return c;
}

// N consecutive entries, in one access of up to 16 bytes
template <class T, int N>
struct alignas(N * sizeof(T)) Pack {
  T x[N];
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(__nv_bfloat16& y, float x) { y = __float2bfloat16(x); }
__device__ __forceinline__ void from_f(__half& y, float x) { y = __float2half(x); }
// the same for two entries of 16 bits in a word
template <class T>
__device__ __forceinline__ float2 unpack(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack<__nv_bfloat16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <>
__device__ __forceinline__ float2 unpack<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
template <class T>
__device__ __forceinline__ uint32_t pack(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&x);
}
template <>
__device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  const __half2 x = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&x);
}

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

// A run of VEC pairs of a head from pair p on.  Pairs from `half` on are the
// entries that are not turned.  Entries stay as they were read until they are used.
template <class T, int VEC, bool INTER>
struct Pairs {
  static constexpr int kWords = VEC == 1 ? 2 : 2 * VEC * (int)sizeof(T) / 4;   // VEC 1: an entry a word
  uint32_t w[kWords];                // first entries, then second ones; INTER: in order
  static __device__ __forceinline__ int lo(int p, int half) { return INTER ? 2 * p : p < half ? p : half + p; }
  static __device__ __forceinline__ int hi(int p, int half, int pairs) { return INTER ? 2 * p + VEC : p < half ? half + p : pairs + p; }
  __device__ __forceinline__ void read(const T* head, int p, int half, int pairs) {
    using W = Pack<uint32_t, kWords / 2>;
    if constexpr (VEC == 1 && sizeof(T) == 2) {
      w[0] = *reinterpret_cast<const uint16_t*>(head + lo(p, half));
      w[1] = *reinterpret_cast<const uint16_t*>(head + hi(p, half, pairs));
    } else {
      *reinterpret_cast<W*>(w) = *reinterpret_cast<const W*>(head + lo(p, half));
      *reinterpret_cast<W*>(w + kWords / 2) = *reinterpret_cast<const W*>(head + hi(p, half, pairs));
    }
  }
  __device__ __forceinline__ void write(T* head, int p, int half, int pairs) const {
    using W = Pack<uint32_t, kWords / 2>;
    if constexpr (VEC == 1 && sizeof(T) == 2) {
      *reinterpret_cast<uint16_t*>(head + lo(p, half)) = (uint16_t)w[0];
      *reinterpret_cast<uint16_t*>(head + hi(p, half, pairs)) = (uint16_t)w[1];
    } else {
      *reinterpret_cast<W*>(head + lo(p, half)) = *reinterpret_cast<const W*>(w);
      *reinterpret_cast<W*>(head + hi(p, half, pairs)) = *reinterpret_cast<const W*>(w + kWords / 2);
    }
  }
  // by the angles of its pairs, which lie at multiples of VEC (widest() below).  WIDE:
  // read four at a time, which saves k_append instructions (with divisions of 64 bits left out, 4 us of 36 for
  // 5595 tokens); k_rope, which waits for memory, takes them one by one (gradient of
  // 8192 tokens of 32 heads of 80: 17.3 us, 19.5 by fours).
  template <bool WIDE>
  __device__ __forceinline__ void by(const float* cosines, const float* sines) {
#pragma unroll
    for (uint32_t& x : w) asm volatile("" : "+r"(x));       // (unpacked from here on, not where they were read)
    constexpr int N = VEC < 4 ? VEC : 4;                    // angles at a time
#pragma unroll
    for (int at = 0; at < VEC; at += N) {
      Pack<float, N> c, s;
      if constexpr (WIDE) {
        c = *reinterpret_cast<const Pack<float, N>*>(cosines + at);
        s = *reinterpret_cast<const Pack<float, N>*>(sines + at);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          c.x[i] = cosines[at + i];
          s.x[i] = sines[at + i];
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 4) {
          uint32_t &u = w[INTER ? 2 * (at + i) : at + i], &v = w[INTER ? 2 * (at + i) + 1 : VEC + at + i];
          float a = __uint_as_float(u), b = __uint_as_float(v);
          turn(a, b, c.x[i], s.x[i]);
          u = __float_as_uint(a);
          v = __float_as_uint(b);
        } else if constexpr (VEC == 1) {
          float a = unpack<T>(w[0]).x, b = unpack<T>(w[1]).x;
          turn(a, b, c.x[0], s.x[0]);
          w[0] = pack<T>(a, 0.f);
          w[1] = pack<T>(b, 0.f);
        } else if constexpr (INTER) {
          float2 x = unpack<T>(w[at + i]);
          turn(x.x, x.y, c.x[i], s.x[i]);
          w[at + i] = pack<T>(x.x, x.y);
        } else if (i % 2 == 0) {
          uint32_t &u = w[(at + i) / 2], &v = w[(VEC + at + i) / 2];
          float2 a = unpack<T>(u), b = unpack<T>(v);
          turn(a.x, b.x, c.x[i], s.x[i]);
          turn(a.y, b.y, c.x[(i + 1) % N], s.x[(i + 1) % N]);
          u = pack<T>(a.x, a.y);
          v = pack<T>(b.x, b.y);
        }
      }
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

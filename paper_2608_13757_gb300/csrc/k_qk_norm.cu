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
#include <cstring>

#include "launch.cuh"
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

// The value of 16 bits in a word
template <class T>
__device__ __forceinline__ float half_word(uint32_t w, bool high) {
  const uint16_t bits = high ? w >> 16 : w & 0xffff;
  T x;
  memcpy(&x, &bits, 2);
  return to_f(x);
}
template <>
__device__ __forceinline__ float half_word<__nv_bfloat16>(uint32_t w, bool high) {
  return __uint_as_float(high ? w & 0xffff0000u : w << 16);
}

// Copies of 8 or 16 bytes from global to shared memory.  A thread closes its
// copies in groups and waits until N groups at most are on their way.
// CACHED where two copies share 32-byte sectors, which then come once.
template <int BYTES, bool CACHED>
__device__ __forceinline__ void copy_ahead(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16 && !CACHED) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int BYTES>
__device__ __forceinline__ void read_shared(uint32_t addr, uint32_t* x) {
  if constexpr (BYTES == 16)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
  else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(addr) : "memory");
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
  static constexpr bool kWide = VECTOR;
  static constexpr int kPiece = VEC * (int)sizeof(T);          // bytes of a wide access: 8 or 16
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
  // A lane's pairs as they were read: in their type where accesses are wide,
  // which takes half the registers until they are used.
  static constexpr bool kRaw = VECTOR && sizeof(T) == 2;
  struct Values {
    uint32_t w[kRaw ? VEC : 2 * VEC];
    __device__ __forceinline__ void clear() {
#pragma unroll
      for (uint32_t& x : w) x = 0;
    }
    // the compiler unpacks again after this instead of keeping what it unpacked
    __device__ __forceinline__ void keep() {
#pragma unroll
      for (uint32_t& x : w) asm volatile("" : "+r"(x));
    }
    __device__ __forceinline__ float operator[](int k) const {
      if constexpr (kRaw) {
        const int e = INTER ? 2 * (k % VEC) + k / VEC : k;
        return half_word<T>(w[e / 2], e % 2);
      } else {
        return __uint_as_float(w[k]);
      }
    }
  };
  __device__ __forceinline__ void read(const T* p, Values& v) const {
    if constexpr (kRaw) {
      struct alignas(2 * VEC) Words {
        uint32_t w[VEC / 2];
      };
      const Words a = *reinterpret_cast<const Words*>(p + lo(0)), b = *reinterpret_cast<const Words*>(p + (INTER ? lo(0) + VEC : hi(0)));
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) { v.w[i] = a.w[i]; v.w[VEC / 2 + i] = b.w[i]; }
    } else {
      float x[2 * VEC] = {};
      read(p, x);
#pragma unroll
      for (int i = 0; i < 2 * VEC; ++i) v.w[i] = __float_as_uint(x[i]);
    }
  }
  __device__ __forceinline__ void read(const T* p, float* x) const {
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
  __device__ __forceinline__ void write(T* p, const float* x) const {
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
  // Wide accesses by way of shared memory: a copy that does not wait, to this
  // lane's place of a slot, and the read when it has come.
  __device__ __forceinline__ void fetch(const T* p, uint32_t slot) const {
    copy_ahead<kPiece, INTER>(slot, p + lo(0));
    copy_ahead<kPiece, INTER>(slot + 32 * kPiece, p + (INTER ? lo(0) + VEC : hi(0)));
  }
  __device__ __forceinline__ void fetched(uint32_t slot, Values& v) const {
    uint32_t y[2 * kPiece / 4];
    read_shared<kPiece>(slot, y);
    read_shared<kPiece>(slot + 32 * kPiece, y + kPiece / 4);
#pragma unroll
    for (int i = 0; i < 2 * kPiece / 4; ++i) v.w[!kRaw && INTER ? i / 2 + i % 2 * VEC : i] = y[i];
  }
  // the angles of a token; NaN for a position outside the table.  Where nothing
  // is rotated no position is looked at: the table may be absent.
  __device__ __forceinline__ void angles(const NormArgs& a, int64_t t, float* c, float* s) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i) { c[i] = 1.f; s[i] = 0.f; }
    if (half == 0) return;
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

// Bytes of a warp's slot for a round of one or two tensors.
template <class S>
constexpr uint32_t kSlot = 2 * 32 * S::kPiece;
template <class S>
constexpr uint32_t kSlot2 = 2 * kSlot<S>;

// A round is the G heads of a token that a warp holds at a time, the queries'
// rounds before the keys'; warps take equal runs of rounds.  One round is
// copied ahead of the one that is computed, in two slots in turn; a lane reads
// only what it copied itself.  Reads in flight without registers are what it
// takes: 16411 tokens of 40 heads of 128 take 56 us (6.1 TB/s) with 80
// registers a thread (24 warps per SM); 59 with 16 warps, 67 with 32, which
// spill.  Read straight into registers by 32 warps a token each: 61.
template <class T, class S>
__global__ void __launch_bounds__(kThreads, 3) k_norm_rope(const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) float part[];   // [kWarps] two slots
  constexpr int VEC = S::VEC, G = 32 / S::LANES;
  const S l(a);
  const int group = (threadIdx.x % 32) / S::LANES;
  const int q_rounds = (a.heads + G - 1) / G, rounds = q_rounds + (a.kv_heads + G - 1) / G;
  const int64_t all = a.rows * rounds, warps = gridDim.x * (int64_t)kWarps, warp = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  int64_t left = all * (warp + 1) / warps - all * warp / warps, t = all * warp / warps / rounds;
  int i = (int)(all * warp / warps - t * rounds);
  int64_t ft = t, fleft = left;
  int fi = i;
  uint32_t slot = 0, both = 0;
  if constexpr (S::kWide) {
    slot = (uint32_t)__cvta_generic_to_shared(part) + threadIdx.x / 32 * 2 * kSlot<S> + threadIdx.x % 32 * S::kPiece;
    both = slot * 2 + kSlot<S>;
  }
  auto fetch = [&] {
    const bool key = fi >= q_rounds;
    const NormTensor& in = key ? a.k : a.q;
    const int h = (key ? fi - q_rounds : fi) * G + group;
    if (fleft > 0 && l.on() && h < (key ? a.kv_heads : a.heads)) l.fetch(static_cast<const T*>(in.data) + ft * in.row + h * in.head, slot);
    end_group();
    --fleft;
    if (++fi == rounds) { fi = 0; ++ft; }
    slot = both - slot;
  };
  if constexpr (S::kWide) fetch();
#pragma unroll 1
  while (left > 0) {
    float c[VEC], s[VEC];
    l.angles(a, t, c, s);
#pragma unroll 1
    while (true) {
      const bool key = i >= q_rounds;
      const int first = key ? q_rounds : 0, n = (int)min(left, (int64_t)(key ? rounds : q_rounds) - i), heads = key ? a.kv_heads : a.heads;
      const NormTensor &in = key ? a.k : a.q, &out = key ? a.k_out : a.q_out;
      float w[2 * VEC];
      l.weights(key ? a.k_weight : a.q_weight, w);
      left -= n;
#pragma unroll 1
      for (const int end = i + n; i < end; ++i) {
        const int h = (i - first) * G + group;
        const bool on = l.on() && h < heads;
        typename S::Values v;
        v.clear();
        if constexpr (S::kWide) {
          fetch();
          wait_groups<1>();
          if (on) l.fetched(slot, v);
        } else if (on) {
          l.read(static_cast<const T*>(in.data) + t * in.row + h * in.head, v);
        }
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) ss += v[e] * v[e];
        const float r = rsqrtf(sum_lanes<S::LANES>(ss) * a.inv_dim + a.eps);
        v.keep();
        float z[2 * VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float p = v[e] * r * w[e], q = v[VEC + e] * r * w[VEC + e];
          z[e] = p * c[e] - q * s[e];
          z[VEC + e] = q * c[e] + p * s[e];
        }
        if (on) l.write(static_cast<T*>(out.data) + t * out.row + h * out.head, z);
      }
      if (left <= 0 || i == rounds) break;
    }
    i = 0;
    ++t;
  }
}

// Gradient, with xh = r x the normed head: dx = r (w dz xh - xh mean(w dz xh)),
// dw = sum of dz xh, dz the output's gradient turned back.  Warps take equal
// runs of rounds, once of the queries and once of the keys; the weights' sums stay in
// registers until the end, go through shared memory in warp order and leave as
// one row per block, so their order does not depend on the run.
// 8192 tokens of 40 heads of 128: 45 us (5.6 TB/s) at 16 warps per SM; the
// angles, weights and sums of a lane take 64 of its 128 registers (80 registers
// for 24 warps: 83).  Whole tokens in turn, 3 or 4 to a warp, took 59, equal
// runs without the copies ahead 55, the next round held in registers 53; two
// and four rounds ahead 48 and 46.
template <class T, class S>
__device__ __forceinline__ void gradient_heads(const NormArgs& a, const S& l, const NormTensor& in, const NormTensor& grad,
                                               const NormTensor& out, int heads, const void* weight, float* row, uint32_t slots) {
  constexpr int VEC = S::VEC, G = 32 / S::LANES;
  const int group = (threadIdx.x % 32) / S::LANES;
  // rounds of G heads, over all tokens, in equal runs
  const int rounds = (heads + G - 1) / G;
  const int64_t all = a.rows * rounds, warps = gridDim.x * (int64_t)kWarps, warp = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  int64_t left = all * (warp + 1) / warps - all * warp / warps, t = all * warp / warps / rounds;
  int h0 = (int)(all * warp / warps - t * rounds) * G;
  float w[2 * VEC], g[2 * VEC];
  l.weights(weight, w);
#pragma unroll
  for (int i = 0; i < 2 * VEC; ++i) g[i] = 0.f;
  // One round ahead of the one that is computed, in two slots in turn.  A lane
  // reads only what it copied itself.
  int64_t ft = t, fleft = left;
  int fh = h0;
  uint32_t slot = slots + threadIdx.x % 32 * S::kPiece;
  const uint32_t both = slot * 2 + kSlot2<S>;
  auto fetch = [&] {
    if (fleft > 0 && l.on() && fh + group < heads) {
      const int h = fh + group;
      l.fetch(static_cast<const T*>(in.data) + ft * in.row + h * in.head, slot);
      l.fetch(static_cast<const T*>(grad.data) + ft * grad.row + h * grad.head, slot + kSlot<S>);
    }
    end_group();
    --fleft;
    fh += G;
    if (fh >= heads) { fh = 0; ++ft; }
    slot = both - slot;
  };
  if constexpr (S::kWide) fetch();
#pragma unroll 1
  for (; left > 0; ++t, h0 = 0) {
    const int h1 = (int)min((int64_t)heads, h0 + left * G);
    left -= (h1 - h0 + G - 1) / G;
    T* dx = static_cast<T*>(out.data) + t * out.row;
    float c[VEC], s[VEC];
    l.angles(a, t, c, s);
#pragma unroll 1
    for (int hb = h0; hb < h1; hb += G) {
      const int h = hb + group;
      const bool on = l.on() && h < h1;
      typename S::Values v, d;
      v.clear();
      d.clear();
      if constexpr (S::kWide) {
        fetch();                          // the next round; the other slot has this one
        wait_groups<1>();
        if (on) {
          l.fetched(slot, v);
          l.fetched(slot + kSlot<S>, d);
        }
      } else if (on) {
        l.read(static_cast<const T*>(in.data) + t * in.row + h * in.head, v);
        l.read(static_cast<const T*>(grad.data) + t * grad.row + h * grad.head, d);
      }
      float ss = 0.f, xd = 0.f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float p = d[i] * c[i] + d[VEC + i] * s[i], q = d[VEC + i] * c[i] - d[i] * s[i];   // turned back
        ss += v[i] * v[i] + v[VEC + i] * v[VEC + i];
        xd += v[i] * p * w[i] + v[VEC + i] * q * w[VEC + i];
      }
      const float r = rsqrtf(sum_lanes<S::LANES>(ss) * a.inv_dim + a.eps);
      const float m = sum_lanes<S::LANES>(xd) * a.inv_dim * r * r;
      if (!on) continue;
      v.keep();
      d.keep();
      float z[2 * VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float p = d[i] * c[i] + d[VEC + i] * s[i], q = d[VEC + i] * c[i] - d[i] * s[i];
        g[i] += p * v[i] * r;
        g[VEC + i] += q * v[VEC + i] * r;
        z[i] = r * (p * w[i] - v[i] * m);
        z[VEC + i] = r * (q * w[VEC + i] - v[VEC + i] * m);
      }
      l.write(dx + h * out.head, z);
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * VEC; ++i)
#pragma unroll
    for (int o = S::LANES; o < 32; o <<= 1) g[i] += __shfl_xor_sync(~0u, g[i], o);
  if (group == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (l.has(i)) {
        row[l.lo(i)] = g[i];
        row[l.hi(i)] = g[VEC + i];
      }
}

template <class T, class S>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope_grad(const __grid_constant__ NormArgs a) {
  extern __shared__ __align__(16) float part[];         // [kWarps][q, k][dim]
  const S l(a);
  float* const row = part + threadIdx.x / 32 * 2 * a.dim;
  uint32_t slots = 0;
  if constexpr (S::kWide)
    slots = (uint32_t)__cvta_generic_to_shared(part + kWarps * 2 * a.dim) + threadIdx.x / 32 * 2 * kSlot2<S>;
  gradient_heads<T>(a, l, a.q, a.q_out, a.dq, a.heads, a.q_weight, row, slots);
  gradient_heads<T>(a, l, a.k, a.k_out, a.dk, a.kv_heads, a.k_weight, row + a.dim, slots);
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * a.dim; e += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += part[w * 2 * a.dim + e];
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + e] = v;
  }
  let_next_start();
}

// The blocks' rows summed in a fixed order: a block takes 32 columns, its
// warps take rows in turn, and the warps' sums are added in warp order.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_weights(const __grid_constant__ NormArgs a, int blocks) {
  __shared__ float part[32][33];
  after_previous();
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
  constexpr int G = 32 / S::LANES;
  const int64_t rounds = a.rows * ((a.heads + G - 1) / G + (a.kv_heads + G - 1) / G), blocks = (rounds + kWarps - 1) / kWarps;
  if (!a.grad) {
    if (a.rows == 0) return cudaSuccess;
    const int n = (int)std::min<int64_t>(blocks, 3 * a.num_sms);
    k_norm_rope<T, S><<<n, kThreads, S::kWide ? kWarps * 2 * kSlot<S> : 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
  }
  const int n = (int)std::min<int64_t>(std::max<int64_t>(1, blocks), norm_blocks(a.num_sms));
  const int shared = kWarps * (2 * a.dim * (int)sizeof(float) + (S::kWide ? 2 * (int)kSlot2<S> : 0));   // 48 KB at most
  k_norm_rope_grad<T, S><<<n, kThreads, shared, st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  count_launch();
  if (!a.q_weight_grad && !a.k_weight_grad) return cudaSuccess;
  e = launch_early(k_norm_weights<T>, (2 * a.dim + 31) / 32, 1024, 0, st, a, n);
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

// Rows into and out of the paged cache (include/sync.h, sync_cache_append and
// sync_cache_read).
//
// Both are one pass over the rows, bound by memory.  A block takes a few tokens;
// a warp per token finds its sequence, its position and its place first, the
// angles are staged in shared memory (rotate.cuh), and the threads then take
// pieces of 16 bytes of the tokens' heads in turn.
#include <algorithm>

#include "cache.h"
#include "paged.cuh"
#include "rotate.cuh"
#include "sync.h"

namespace syncgb {
namespace {

using namespace rotate;

constexpr int kThreads = 256, kTokens = 8;       // most tokens of a block: one per warp
constexpr int kAhead = 4;                        // pieces that a thread reads before it writes the first

// 8 entries of a row, by one access or entry by entry
template <class T>
__device__ __forceinline__ void load8(const T* p, bool wide, float* x) {
  if (wide) {
    const Pack<T, 8> v = *reinterpret_cast<const Pack<T, 8>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f(v.x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f(p[i]);
  }
}

// Entries d .. d + 7 of a key head after the rotation.  c: cosines of the
// token's pairs, then its sines.
template <class T>
__device__ __forceinline__ void turned8(const T* head, int d, bool wide, int half, bool interleaved, const float* c, float* x) {
  const float* s = c + half;
  if (interleaved) {
    load8(head + d, wide, x);
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      if (d + i < 2 * half) turn(x[i], x[i + 1], c[(d + i) / 2], s[(d + i) / 2]);
  } else if (wide && half % 8 == 0) {
    load8(head + d, wide, x);
    if (d >= 2 * half) return;
    float y[8];
    const int j = d < half ? d : d - half;
    load8(head + (d < half ? d + half : j), wide, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (d < half) turn(x[i], y[i], c[j + i], s[j + i]);
      else turn(y[i], x[i], c[j + i], s[j + i]);
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      const int e = d + i, j = e < half ? e : e - half;
      float v = to_f(head[e]);
      if (e < 2 * half) {
        float u = to_f(head[e < half ? e + half : j]);
        if (e < half) turn(v, u, c[j], s[j]);
        else turn(u, v, c[j], s[j]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = k == i ? v : x[k];
    }
  }
}

// 8 entries as 4-bit codes, with the scale of their group, which four
// consecutive lanes share: scale = max |x| / 7 rounded to float16, code =
// x / scale rounded to even, at most 7 in size, stored plus 8.  The divisions
// are by the scale as it is kept.  A group with a NaN or an infinity reads as
// NaN, one beyond 7 * 65504 ends at that.
__device__ __forceinline__ uint32_t codes8(const float* x, __half& scale, uint32_t lanes) {
  uint32_t top = 0;                                         // as bits, so that a NaN is the largest
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(lanes, top, 1));
  top = max(top, __shfl_xor_sync(lanes, top, 2));
  scale = top >= 0x7f800000u ? __ushort_as_half(0x7fff) : __float2half(fminf(__fdiv_rn(__uint_as_float(top), 7.f), 65504.f));
  const float by = __half2float(scale);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int code = by > 0.f ? min(7, max(-7, __float2int_rn(__fdiv_rn(x[i], by)))) : 0;
    word |= (uint32_t)(code + 8) << (4 * i);
  }
  return word;
}

// New tokens into the cache.  T: their type.  QVEC: pairs of a query head that
// a thread takes at a time.
template <class T, int QVEC, bool INTER>
__global__ void __launch_bounds__(kThreads) k_append(const __grid_constant__ CacheArgs a, int tokens, bool kv_wide) {
  extern __shared__ __align__(16) float angles[];           // [tokens][cos, sin][half]
  __shared__ int64_t place[kTokens], pos[kTokens];
  __shared__ bool mine[kTokens];                            // a sequence has the row
  const int half = a.turn.half, warp = threadIdx.x / 32;
  const int64_t row0 = blockIdx.x * (int64_t)tokens;
  const int n = (int)min((int64_t)tokens, a.rows - row0);
  if (warp < n) {
    const int64_t row = row0 + warp;
    const int s = paged::sequence_of(a, row);
    if (threadIdx.x % 32 == 0) {
      int64_t at = -1;
      if (s >= 0) at = a.starts ? (int64_t)__ldg(a.lens + s) - __ldg(a.starts + s + 1) + row : (int64_t)__ldg(a.lens + s) - 1;
      mine[warp] = s >= 0;
      pos[warp] = at;
      place[warp] = s >= 0 ? paged::place_of(a, s, at) : -1;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int t = i / half, j = i - t * half;
    if (!mine[t]) continue;
    const float2 x = angle(a.turn, position(a.turn, row0 + t, pos[t], j), j);
    angles[2 * t * half + j] = x.x;
    angles[(2 * t + 1) * half + j] = x.y;
  }
  __syncthreads();
  if (a.heads) {                                            // queries, as k_rope turns them
    const int pairs = a.dim / 2;
    Walk w(threadIdx.x, kThreads, a.heads, pairs / QVEC);
    while (w.t < n) {
      Pairs<T, QVEC, INTER> x[kAhead];
      Walk at = w;
#pragma unroll
      for (int e = 0; e < kAhead; ++e, at.next()) {
        if (at.t >= n) break;
        if (mine[at.t]) x[e].read(static_cast<const T*>(a.q.data) + (row0 + at.t) * a.q.row + at.h * a.q.head, at.r * QVEC, half, pairs);
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e, w.next()) {
        if (w.t >= n) break;
        const int p = w.r * QVEC;
        if (!mine[w.t]) {
          if (!a.fill) continue;
#pragma unroll
          for (int i = 0; i < 2 * QVEC; ++i) from_f(x[e].x[i], 0.f);
        } else if (p < half) {
          const float* c = angles + 2 * w.t * half + p;
          x[e].by(c, c + half);
        }
        x[e].write(static_cast<T*>(a.q_out.data) + (row0 + w.t) * a.q_out.row + w.h * a.q_out.head, p, half, pairs);
      }
    }
  }
  // keys, then values: 8 entries per thread
  // (a row has a multiple of 4 runs where the cache has 4 bits: the lanes of a group agree)
  const int g = a.dim / kGroup;
  for (Walk w(threadIdx.x, kThreads, 2 * a.kv_heads, a.dim / 8); w.t < n; w.next()) {
    const int t = w.t, e = w.r, d = 8 * e;
    if (place[t] < 0) continue;
    const bool is_v = w.h >= a.kv_heads;
    const int h = is_v ? w.h - a.kv_heads : w.h;
    const HeadTensor& in = is_v ? a.v_rows : a.k_rows;
    const T* head = static_cast<const T*>(in.data) + (row0 + t) * in.row + h * in.head;
    const int64_t at = paged::row_of(a, place[t], h);
    float x[8];
    if (is_v) load8(head + d, kv_wide, x);
    else turned8(head, d, kv_wide, half, INTER, angles + 2 * t * half, x);
    if (a.bits == 16) {
      Pack<T, 8> y;
#pragma unroll
      for (int k = 0; k < 8; ++k) from_f(y.x[k], x[k]);
      *reinterpret_cast<Pack<T, 8>*>((is_v ? a.v : a.k) + (at * a.dim + d) * 2) = y;
    } else {
      __half scale;
      const uint32_t word = codes8(x, scale, 0xfu << (threadIdx.x % 32 / 4 * 4));
      *reinterpret_cast<uint32_t*>((is_v ? a.v : a.k) + at * (a.dim / 2) + 4 * paged::word_of(e, g)) = word;
      if (e % 4 == 0) reinterpret_cast<__half*>(is_v ? a.v_scale : a.k_scale)[at * g + e / 4] = scale;
    }
  }
}

// Cached tokens back to rows of 16 bits: the tokens of sequence s from its first
// one on go to rows starts[s] .. starts[s + 1]; zeros past its length.
template <class T>
__global__ void __launch_bounds__(kThreads) k_read(const __grid_constant__ CacheArgs a, int tokens) {
  __shared__ int64_t place[kTokens];                        // -1: no such token, -2: not a sequence's row, -3: no such page
  const int64_t row0 = blockIdx.x * (int64_t)tokens;
  const int n = (int)min((int64_t)tokens, a.rows - row0), warp = threadIdx.x / 32;
  if (warp < n) {
    const int64_t row = row0 + warp;
    const int s = paged::sequence_of(a, row);
    if (threadIdx.x % 32 == 0) {
      int64_t at = -2;
      if (s >= 0) {
        const int64_t p = row - (a.starts ? __ldg(a.starts + s) : row);
        at = p < __ldg(a.lens + s) ? paged::place_of(a, s, p) : -1;
        if (at < 0 && p < __ldg(a.lens + s)) at = -3;
      }
      place[warp] = at;
    }
  }
  __syncthreads();
  const int g = a.dim / kGroup;
  Walk w(threadIdx.x, kThreads, 2 * a.kv_heads, a.dim / 8);
  while (w.t < n) {
    Pack<T, 8> y[kAhead];                                   // 16 bits: the entries; 4: a word of codes and its scale
    Walk at = w;
#pragma unroll
    for (int e = 0; e < kAhead; ++e, at.next()) {
      if (at.t >= n) break;
      if (place[at.t] < 0) continue;
      const bool is_v = at.h >= a.kv_heads;
      const int64_t row = paged::row_of(a, place[at.t], is_v ? at.h - a.kv_heads : at.h);
      if (a.bits == 16) {
        y[e] = *reinterpret_cast<const Pack<T, 8>*>((is_v ? a.v : a.k) + (row * a.dim + 8 * at.r) * 2);
      } else {
        uint32_t* in = reinterpret_cast<uint32_t*>(&y[e]);
        in[0] = __ldg(reinterpret_cast<const uint32_t*>((is_v ? a.v : a.k) + row * (a.dim / 2)) + paged::word_of(at.r, g));
        in[1] = __ldg(reinterpret_cast<const uint16_t*>(is_v ? a.v_scale : a.k_scale) + row * g + at.r / 4);
      }
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e, w.next()) {
      if (w.t >= n) break;
      const int64_t from = place[w.t];
      if (from == -2 && !a.fill) continue;
      if (from < 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) from_f(y[e].x[k], from == -3 ? __int_as_float(0x7fffffff) : 0.f);
      } else if (a.bits == 4) {
        const uint32_t* in = reinterpret_cast<const uint32_t*>(&y[e]);
        const uint32_t word = in[0];
        const float scale = __half2float(__ushort_as_half((uint16_t)in[1]));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float x = (float)((int)(word >> (4 * k) & 15) - 8) * scale;
          // 7 scales may be past float16's end where the row's largest entry was not: the scale was rounded
          if (!a.bf16) x = x > 65504.f ? 65504.f : x < -65504.f ? -65504.f : x;
          from_f(y[e].x[k], x);
        }
      }
      const bool is_v = w.h >= a.kv_heads;
      const HeadTensor& out = is_v ? a.v_rows : a.k_rows;
      *reinterpret_cast<Pack<T, 8>*>(static_cast<T*>(out.data) + (row0 + w.t) * out.row + (is_v ? w.h - a.kv_heads : w.h) * out.head + 8 * w.r) = y[e];
    }
  }
}

// Tokens of a block: enough for its threads to have several pieces in flight,
// as long as every SM has blocks.
int tokens_of(int64_t rows, int num_sms) { return (int)std::max<int64_t>(1, std::min<int64_t>(kTokens, rows / (4 * num_sms))); }

template <class T, int QVEC>
cudaError_t append(const CacheArgs& a, bool kv_wide, cudaStream_t st) {
  const int tokens = tokens_of(a.rows, a.num_sms);
  const unsigned blocks = (unsigned)((a.rows + tokens - 1) / tokens);
  const size_t smem = (size_t)tokens * 2 * a.turn.half * sizeof(float);
  if (a.turn.interleaved) k_append<T, QVEC, true><<<blocks, kThreads, smem, st>>>(a, tokens, kv_wide);
  else k_append<T, QVEC, false><<<blocks, kThreads, smem, st>>>(a, tokens, kv_wide);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

template <class T>
cudaError_t append_type(const CacheArgs& a, cudaStream_t st) {
  bool wide = true;
  for (const HeadTensor* t : {&a.k_rows, &a.v_rows})
    wide = wide && reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->row % 8 == 0 && t->head % 8 == 0;
  const HeadTensor q[2] = {a.q, a.q_out};
  const int vec = a.heads ? widest(q, 2, 2, a.turn.half, a.dim) : 8;
  if (vec == 8) return append<T, 8>(a, wide, st);
  if (vec == 4) return append<T, 4>(a, wide, st);
  return append<T, 1>(a, wide, st);
}

}  // namespace

cudaError_t launch_cache_append(const CacheArgs& a, cudaStream_t st) {
  if (!a.rows) return cudaSuccess;
  return a.bf16 ? append_type<__nv_bfloat16>(a, st) : append_type<__half>(a, st);
}

cudaError_t launch_cache_read(const CacheArgs& a, cudaStream_t st) {
  if (!a.rows) return cudaSuccess;
  const int tokens = tokens_of(a.rows, a.num_sms);
  const unsigned blocks = (unsigned)((a.rows + tokens - 1) / tokens);
  if (a.bf16) k_read<__nv_bfloat16><<<blocks, kThreads, 0, st>>>(a, tokens);
  else k_read<__half><<<blocks, kThreads, 0, st>>>(a, tokens);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace syncgb

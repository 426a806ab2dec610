// Rotation of query and key heads by positions with up to four axes
// (include/sync.h, sync_rope), and its gradient, which is the rotation by minus
// the angles.
//
// One pass, bound by memory: an entry is read and written once.  A block takes
// a few tokens; its threads take runs of pairs of all their heads in turn,
// kAhead at a time, so that every thread has two wide reads per run in flight.
#include <algorithm>

#include "cache.h"
#include "rotate.cuh"
#include "sync.h"

namespace syncgb {
namespace {

using namespace rotate;

constexpr int kThreads = 256, kAhead = 4;

template <class T, int VEC, bool INTER>
__global__ void __launch_bounds__(kThreads) k_rope(const __grid_constant__ RopeArgs a, int tokens) {
  extern __shared__ __align__(16) float angles[];          // [tokens][cos, sin][half]
  const int half = a.turn.half, pairs = a.dim / 2, runs = pairs / VEC, heads = a.heads + a.kv_heads;
  const int64_t row0 = blockIdx.x * (int64_t)tokens;
  const int n = (int)min((int64_t)tokens, a.rows - row0);
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int t = i / half, j = i - t * half;
    const float2 x = angle(a.turn, position(a.turn, row0 + t, row0 + t, j), j);
    angles[2 * t * half + j] = x.x;
    angles[(2 * t + 1) * half + j] = x.y;
  }
  __syncthreads();
  const int each = heads * runs, all = n * each;
  for (int i0 = threadIdx.x; i0 < all; i0 += kAhead * kThreads) {
    Pairs<T, VEC, INTER> x[kAhead];
    T* to[kAhead];
    int p[kAhead], t[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int i = i0 + e * kThreads;
      if (i >= all) break;
      t[e] = i / each;
      const int r = i - t[e] * each, h = r / runs;
      p[e] = (r - h * runs) * VEC;
      const bool is_q = h < a.heads;
      const HeadTensor &in = is_q ? a.q : a.k, &out = is_q ? a.q_out : a.k_out;
      const int64_t row = row0 + t[e], head = is_q ? h : h - a.heads;
      to[e] = static_cast<T*>(out.data) + row * out.row + head * out.head;
      x[e].read(static_cast<const T*>(in.data) + row * in.row + head * in.head, p[e], half, pairs);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (i0 + e * kThreads >= all) break;
      const float* c = angles + 2 * t[e] * half + p[e];
      if (p[e] < half) x[e].by(c, c + half);
      x[e].write(to[e], p[e], half, pairs);
    }
  }
}

template <class T, int VEC>
cudaError_t launch(const RopeArgs& a, cudaStream_t st) {
  // enough tokens for every thread to have its runs in flight, as long as every SM has a block
  const int64_t each = (int64_t)(a.heads + a.kv_heads) * (a.dim / 2 / VEC);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(8, kAhead * kThreads / std::max<int64_t>(1, each)));
  const int tokens = (int)std::max<int64_t>(1, std::min<int64_t>(want, a.rows / (2 * a.num_sms)));
  const unsigned blocks = (unsigned)((a.rows + tokens - 1) / tokens);
  const size_t smem = (size_t)tokens * 2 * a.turn.half * sizeof(float);
  if (a.turn.interleaved) k_rope<T, VEC, true><<<blocks, kThreads, smem, st>>>(a, tokens);
  else k_rope<T, VEC, false><<<blocks, kThreads, smem, st>>>(a, tokens);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

template <class T>
cudaError_t launch_type(const RopeArgs& a, cudaStream_t st) {
  const HeadTensor all[4] = {a.q, a.k, a.q_out, a.k_out};
  const int vec = widest(all, 4, (int)sizeof(T), a.turn.half, a.dim);
  if (vec * sizeof(T) == 16) return launch<T, 16 / sizeof(T)>(a, st);
  if (vec * sizeof(T) == 8) return launch<T, 8 / sizeof(T)>(a, st);
  return launch<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  if (!a.rows) return cudaSuccess;
  if (a.dtype == SYNC_BF16) return launch_type<__nv_bfloat16>(a, st);
  if (a.dtype == SYNC_FP16) return launch_type<__half>(a, st);
  return launch_type<float>(a, st);
}

}  // namespace syncgb

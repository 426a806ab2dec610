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
__global__ void __launch_bounds__(kThreads, 3) k_rope(const __grid_constant__ RopeArgs a, int tokens) {
  extern __shared__ __align__(16) float angles[];          // [tokens][cos, sin][half]
  const int half = a.turn.half, pairs = a.dim / 2, heads = a.heads + a.kv_heads;
  const int64_t row0 = blockIdx.x * (int64_t)tokens;
  const int n = (int)min((int64_t)tokens, a.rows - row0);
  Walk w(threadIdx.x, kThreads, heads, pairs / VEC);
  Pairs<T, VEC, INTER> x[kAhead];
  auto read = [&](Walk at) {                                // the next runs
#pragma unroll
    for (int e = 0; e < kAhead; ++e, at.next()) {
      if (at.t >= n) break;
      const HeadTensor& in = at.h < a.heads ? a.q : a.k;
      x[e].read(static_cast<const T*>(in.data) + (row0 + at.t) * in.row + (at.h < a.heads ? at.h : at.h - a.heads) * in.head,
                at.r * VEC, half, pairs);
    }
  };
  read(w);                                                  // under the way to the angles
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int t = i / half, j = i - t * half;
    const float2 y = angle(a.turn, position(a.turn, row0 + t, row0 + t, j), j);
    angles[2 * t * half + j] = y.x;
    angles[(2 * t + 1) * half + j] = y.y;
  }
  __syncthreads();
  while (w.t < n) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e, w.next()) {
      if (w.t >= n) break;
      const int p = w.r * VEC;
      const float* c = angles + 2 * w.t * half + p;
      if (p < half) x[e].by(c, c + half);
      const HeadTensor& out = w.h < a.heads ? a.q_out : a.k_out;
      x[e].write(static_cast<T*>(out.data) + (row0 + w.t) * out.row + (w.h < a.heads ? w.h : w.h - a.heads) * out.head, p, half, pairs);
    }
    if (w.t < n) read(w);
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

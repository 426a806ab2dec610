// Rotation of query and key heads by positions with up to four axes
// (include/sync.h, sync_rope), and its gradient, which is the rotation by minus
// the angles.
//
// One pass, bound by memory: an entry is read and written once (rotate.cuh says
// how).  16411 tokens of 40 heads of 128 entries with three axes take 56 us,
// 6.2 TB/s (a plain copy 6.8); 92 with the angles staged in front of each group
// instead of under the one before.
#include "cache.h"
#include "rotate.cuh"
#include "sync.h"

namespace syncgb {
namespace {

using namespace rotate;

template <class T, int VEC, bool INTER>
__global__ void __launch_bounds__(kResident, 1) k_rope(const __grid_constant__ RopeArgs a, const __grid_constant__ Columns c) {
  extern __shared__ __align__(16) float angles[];          // [2][tokens][cos, sin][half]
  const int half = a.turn.half, pairs = a.dim / 2, runs = pairs / VEC, tokens = c.tokens();
  const int sub = threadIdx.x / c.each, column = blockIdx.y * c.each + threadIdx.x % c.each;
  const bool on = sub < c.par && column < (a.heads + a.kv_heads) * runs;
  const int h = column / runs, p = (column - h * runs) * VEC;
  const bool is_q = h < a.heads;
  const HeadTensor &in = is_q ? a.q : a.k, &out = is_q ? a.q_out : a.k_out;
  const T* const from = static_cast<const T*>(in.data) + (is_q ? h : h - a.heads) * in.head;
  T* const to = static_cast<T*>(out.data) + (is_q ? h : h - a.heads) * out.head;
  const int64_t in_row = in.row, out_row = out.row;

  Pairs<T, VEC, INTER> x[kAhead];
  auto read = [&](int64_t group) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int64_t row = group * tokens + sub + e * c.par;
      if (on && e < c.ahead && row < a.rows) x[e].read(from + row * in_row, p, half, pairs);
    }
  };
  // staged entries of this thread: pair j of token t
  int t[kStaged], j[kStaged], pos[kStaged];
  float2 turned[kStaged];
#pragma unroll
  for (int e = 0; e < kStaged; ++e) {
    const int i = threadIdx.x + e * blockDim.x;
    t[e] = i < tokens * half ? i / half : -1;
    j[e] = i - t[e] * half;
  }
  auto look = [&](int64_t group) {                          // positions of a group
#pragma unroll
    for (int e = 0; e < kStaged; ++e) {
      const int64_t row = group * tokens + t[e];
      pos[e] = t[e] >= 0 && row < a.rows ? (int)position(a.turn, row, row, j[e]) : 0;
    }
  };
  auto find = [&] {                                         // and their angles
#pragma unroll
    for (int e = 0; e < kStaged; ++e)
      if (t[e] >= 0) turned[e] = angle(a.turn, pos[e], j[e]);
  };
  auto put = [&](int which) {
#pragma unroll
    for (int e = 0; e < kStaged; ++e)
      if (t[e] >= 0) {
        float* at = angles + ((which * tokens + t[e]) * 2) * half + j[e];
        at[0] = turned[e].x;
        at[half] = turned[e].y;
      }
  };
  int64_t group = blockIdx.x;
  read(group);
  look(group);
  find();
  put(0);
  look(group + gridDim.x);
  __syncthreads();
  for (int which = 0; group < c.groups; which ^= 1) {
    const int64_t next = group + gridDim.x;
    if (next < c.groups) find();
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int token = sub + e * c.par;
      const int64_t row = group * tokens + token;
      if (on && e < c.ahead && row < a.rows) {
        const float* cs = angles + ((which * tokens + token) * 2) * half + p;
        if (p < half) x[e].template by<false>(cs, cs + half);
        x[e].write(to + row * out_row, p, half, pairs);
      }
    }
    if (next < c.groups) {
      read(next);
      put(which ^ 1);
      look(next + gridDim.x);
    }
    group = next;
    __syncthreads();
  }
}

template <class T, int VEC>
cudaError_t launch(const RopeArgs& a, cudaStream_t st) {
  const Columns c = columns_of(a.rows, (a.heads + a.kv_heads) * (a.dim / 2 / VEC), kAhead, a.turn.half, a.num_sms);
  const dim3 grid((unsigned)c.blocks_x, (unsigned)c.blocks_y);
  const size_t smem = (size_t)4 * c.tokens() * a.turn.half * sizeof(float);
  if (a.turn.interleaved) k_rope<T, VEC, true><<<grid, c.threads, smem, st>>>(a, c);
  else k_rope<T, VEC, false><<<grid, c.threads, smem, st>>>(a, c);
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

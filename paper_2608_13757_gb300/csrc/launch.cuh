// Launches of kernels that follow one another in a call.
#pragma once

#include <cuda_runtime.h>

namespace syncgb {

// In a kernel: waits until the kernels before it in its stream are done and
// their writes are visible (at once where it was launched in the plain way).
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// In a kernel: one that launch_early() puts behind it may start.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launches a kernel that may start before its predecessor in the stream is
// done, as soon as every block of that one has called let_next_start() and
// there is room; it calls after_previous() before it uses its results, and
// before it ends.  What it reads or writes before after_previous() must be safe
// while its predecessor runs, outputs as well as inputs: their memory may be
// what the predecessor still reads.  And the predecessor has to be a known one:
// of the work before that, only what the predecessor itself waited for is done.
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = grid;
  c.blockDim = block;
  c.dynamicSmemBytes = smem;
  c.stream = st;
  c.attrs = &early;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, args...);
}

// Launches a kernel behind all earlier work of the stream.
template <class... P, class... A>
cudaError_t launch_plain(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const A&... args) {
  kernel<<<grid, block, smem, st>>>(args...);
  return cudaGetLastError();
}

}  // namespace syncgb

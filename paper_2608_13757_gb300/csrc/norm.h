// Head norms with the position rotation: what the C ABI passes to k_qk_norm.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace syncgb {

void count_launch();

struct NormTensor {
  void* data = nullptr;
  int64_t row = 0, head = 0;     // strides in entries
};

struct NormArgs {
  int dtype = 0;                 // sync_dtype
  bool grad = false;
  int heads = 0, kv_heads = 0, dim = 0, rotated = 0;
  bool interleaved = false;
  float eps = 0.f, inv_dim = 0.f;
  int64_t rows = 0, n_positions = 0;
  NormTensor q, k;               // inputs
  NormTensor q_out, k_out;       // outputs; with grad, their gradients
  NormTensor dq, dk;
  const void *q_weight = nullptr, *k_weight = nullptr;
  void *q_weight_grad = nullptr, *k_weight_grad = nullptr;
  const float *cos = nullptr, *sin = nullptr;
  const int32_t* positions = nullptr;
  float* partial = nullptr;      // [norm_blocks][q, k][dim]
  int num_sms = 0;
};

// Most blocks of the gradient kernel: two per SM, which keeps every SM full.
inline int norm_blocks(int num_sms) { return 2 * num_sms; }

cudaError_t launch_norm_rope(const NormArgs& a, cudaStream_t st);

}  // namespace syncgb

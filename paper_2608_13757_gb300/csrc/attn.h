// Attention over packed sequences: the plan, and what the C ABI passes to the
// kernels (k_attn_fwd.cu, k_attn_bwd.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <vector>

#include "sync.h"

namespace syncgb {

void count_launch();

constexpr int kTile = 128;         // rows of a query tile and of a key tile

struct AttnSeq {
  int64_t q0, k0;                  // first rows in the query and key tensors
  int32_t lq, lk;
};

// A query tile of one head, or a key tile of one key head.
struct AttnItem {
  int32_t seq, head, tile, pad;
};

struct AttnTensor {
  void* data = nullptr;
  int64_t rows = 0, row = 0, head = 0;   // strides in entries
};

struct AttnArgs {
  bool bf16 = true;
  int heads = 0, kv_heads = 0, dim = 0;
  float scale = 0.f;
  const AttnSeq* seq = nullptr;
  AttnTensor q, k, v, o, d_o, dq, dk, dv;
  float* lse = nullptr;            // [heads][q.rows]
  float* delta = nullptr;          // [heads][delta_rows], the plan's
  int64_t delta_rows = 0;
  const AttnItem *q_item = nullptr, *k_item = nullptr;
  int n_q_items = 0, n_k_items = 0;
  int num_sms = 0;
};

cudaError_t launch_attn_forward(const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attn_backward(const AttnArgs& a, cudaStream_t st);

}  // namespace syncgb

struct sync_attn {
  int device = 0, num_sms = 0;
  bool train = false;
  sync_attn_sizes sz{};
  syncgb::AttnArgs args;           // sizes and device tables
  std::vector<void*> blocks;
};

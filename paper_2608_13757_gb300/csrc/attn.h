// Attention over packed sequences: the plan, and what the C ABI passes to the
// kernels (k_attn_fwd.cu, k_attn_bwd.cu).
#pragma once

#include <cuda.h>
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

// A forward item: two consecutive query tiles of a sequence against the key
// tiles [kt0, kt1).  A tile's rows are 128 queries of one head, or (packed)
// the queries' heads of a group, 128 / group queries.
struct AttnItem {
  int32_t seq, head, q0, packed;   // head: the first one of a packed tile
  int32_t kt0, kt1;
  int32_t group, piece;            // a split key range: which, and its piece; group -1: whole
};

// A split key range: its pieces' results are at slot, slot + 1, ...
struct AttnSplit {
  int32_t slot, pieces;
};

// A query tile of one head, or a key tile of one key head (gradients).
struct AttnTile {
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
  // forward: items of block b are item[block_first[b] .. block_first[b + 1])
  const AttnItem* item = nullptr;
  const int32_t* block_first = nullptr;
  int n_blocks = 0;
  const AttnSplit* split = nullptr;
  int32_t* split_count = nullptr;  // [splits][2]: pieces that are done
  float *part_o = nullptr, *part_lse = nullptr;   // [slots][2][kTile](dim padded), [slots][2][kTile]
  // gradients: tiles of block b are tile[first[b] .. first[b + 1])
  const AttnTile *q_tile = nullptr, *k_tile = nullptr;
  const int32_t *q_first = nullptr, *k_first = nullptr;
  int n_q_blocks = 0, n_k_blocks = 0;
  int* error = nullptr;            // host-visible: a kernel gave up waiting
  int num_sms = 0;
};

// Tiles of the tensors as TMA loads them: 64 entries by 128 rows of one head;
// q_group by the heads of a group.
struct AttnMaps {
  CUtensorMap q, q_group, k, v, d_o;
};

cudaError_t launch_attn_forward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st);
cudaError_t launch_attn_backward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st);

}  // namespace syncgb

struct sync_attn {
  int device = 0, num_sms = 0;
  bool train = false;
  sync_attn_sizes sz{};
  syncgb::AttnArgs args;           // sizes and device tables
  void* block = nullptr;           // device memory
  int* error = nullptr;            // pinned
};

// Attention over packed sequences: the plan, and what the C ABI passes to the
// kernels (k_attn_fwd.cu, k_attn_bwd.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <vector>

#include "cache.h"
#include "sync.h"

namespace syncgb {

void count_launch();

constexpr int kTile = 128;         // rows of a query tile and of a key tile

// A forward item: two consecutive query tiles of a sequence against a range of
// key tiles.  A tile's rows are 128 queries of one head, or (packed) the
// queries' heads of a group, 128 / group queries.  Everything a block needs to
// know is in these 64 bytes, so that an item costs one access.
struct alignas(64) AttnItem {
  int64_t q_row, k_row;            // rows of the tensors: first query, first key of the range
  int32_t head, packed;            // head: the first one of a packed tile
  int32_t rows[2];                 // queries of each tile
  int32_t n[2];                    // key tiles that each meets
  int32_t seen;                    // keys of the range that the first query sees (may be negative); the next sees one more
  int32_t keys;                    // keys of the sequence from k_row on
  int32_t slot;                    // where a piece of a split range leaves its result; -1: the range is whole
};

// A split key range: its pieces' results are at slot, slot + 1, ...
struct AttnSplit {
  int64_t q_row;
  int32_t head, packed, rows[2], slot, pieces;
};

// A gradient item.  Key walk: a key tile of a key head against n query tiles
// of each head of its group, from q_row on.  Query walk: a query tile of a
// head against n key tiles from k_row on.
struct alignas(64) AttnTile {
  int64_t q_row, k_row;
  int32_t head, n;
  int32_t rows, keys;              // queries from q_row on and keys from k_row on that are the sequence's
  int32_t seen;                    // keys from k_row on that the query at q_row sees (may be negative)
};

struct AttnTensor {
  void* data = nullptr;
  int64_t rows = 0, row = 0, head = 0;   // strides in entries
};

struct AttnArgs {
  bool bf16 = true;
  int heads = 0, kv_heads = 0, dim = 0;
  float scale = 0.f;
  AttnTensor q, k, v, o, d_o, dq, dk, dv;
  float* lse = nullptr;            // [heads][q.rows]
  float* delta = nullptr;          // [heads][delta_rows], the plan's
  int64_t delta_rows = 0;
  // forward: items of block b are item[block_first[b] .. block_first[b + 1])
  const AttnItem* item = nullptr;
  const int32_t* block_first = nullptr;
  int n_blocks = 0;
  const AttnSplit* split = nullptr;
  int n_splits = 0, merge_rows = 0;               // most rows of a split range
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
cudaError_t launch_wait_in_vain(int* error, int tries, cudaStream_t st);   // for tests

}  // namespace syncgb

struct sync_attn {
  int device = 0, num_sms = 0;
  bool train = false;
  sync_attn_sizes sz{};
  syncgb::AttnArgs args;           // sizes and device tables
  bool few = false;                // few queries per sequence: k_cache_attn.cu, and what it takes
  syncgb::CacheArgs rows;
  void* block = nullptr;           // device memory
  int* error = nullptr;            // pinned
};

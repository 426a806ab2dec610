// Rotation by several axes and the paged cache: what the C ABI (cache.cpp)
// passes to the kernels (k_rope.cu, k_cache.cu, k_cache_attn.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace syncgb {

void count_launch();

constexpr int kAxes = 4, kMostPairs = 128;
constexpr int kGroup = 32;           // entries that share a scale in 4 bits

struct HeadTensor {
  void* data = nullptr;
  int64_t rows = 0, row = 0, head = 0;   // strides in entries
};

struct Rotation {
  int half = 0;                      // pairs that are turned
  bool interleaved = false;
  float way = 1.f;                   // -1: by minus the angles
  const float *cos = nullptr, *sin = nullptr;
  int64_t n_positions = 0;
  const int32_t* positions = nullptr;
  int64_t position_stride = 0;
  uint32_t axis[kMostPairs / 16] = {};   // two bits for each pair
};

struct RopeArgs {
  int dtype = 0;                     // sync_dtype
  int heads = 0, kv_heads = 0, dim = 0;
  int64_t rows = 0;
  HeadTensor q, k, q_out, k_out;
  Rotation turn;
  int num_sms = 0;
};

// The cache and the sequences of a step.
struct CacheArgs {
  bool bf16 = true;
  int bits = 16, kv_heads = 0, dim = 0, page_shift = 0, n_pages = 0;
  uint8_t *k = nullptr, *v = nullptr;          // [pages][kv_heads][page] rows
  uint8_t *k_scale = nullptr, *v_scale = nullptr;
  int n_seqs = 0, max_pages = 0;
  const int32_t* table = nullptr;
  int64_t table_stride = 0;
  const int32_t *lens = nullptr, *starts = nullptr;
  int64_t rows = 0;                            // of the tensors
  bool fill = false;                           // rows that no sequence has become zero
  int num_sms = 0;
  // append: new rows; read: where they go
  HeadTensor k_rows, v_rows;
  // append and attention
  int heads = 0;
  HeadTensor q, q_out;
  Rotation turn;
  // attention
  float scale = 0.f;
  float* lse = nullptr;                        // [heads][rows]
  int most_rows = 1;                           // query rows of a key head that a pass takes: 8, 16, 32
  int blocks = 0;
  uint8_t* work = nullptr;
  bool whole = false;                          // no pass is cut between warps
  // attention of few queries over plain rows: sequence s has rows starts[s] and on,
  // counts[s] of them, and lens[s] keys from row firsts[s] of k_rows and v_rows on,
  // all of which they see
  const int32_t* counts = nullptr;
  const int64_t* firsts = nullptr;
};

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st);
cudaError_t launch_cache_append(const CacheArgs& a, cudaStream_t st);
cudaError_t launch_cache_read(const CacheArgs& a, cudaStream_t st);
cudaError_t launch_cache_attn(const CacheArgs& a, cudaStream_t st);
cudaError_t launch_few_queries(const CacheArgs& a, cudaStream_t st);

// Blocks and workspace of an attention call, at a multiple of kWorkAlign bytes.
constexpr int kWorkAlign = 16;
int cache_attn_rows(int bits, int group, int max_new);                // query rows of a pass: 8, 16, 32
int cache_attn_blocks(int bits, int most_rows, int num_sms);
int64_t cache_attn_workspace(int dim, int most_rows, int blocks);

}  // namespace syncgb

// Gradients of attention over packed sequences (include/sync.h,
// sync_attn_backward), with P = exp(S - lse) recomputed from the scores:
//   delta = rowsum(O dO),  dS = P (dO V^T - delta),
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
//
// Three kernels: delta, one that walks query tiles for a key tile (dK, dV),
// and one that walks key tiles for a query tile (dQ).  Adding dQ up from the
// first walk would save recomputing S and dO V^T (5 products instead of 7),
// but by atomic additions in 32 bits, whose order, and with it the result,
// changes from run to run, and which cost a read and a write of dQ in L2 for
// every pair of tiles.
//
// A walk takes one block per SM, tiles of 128 by 128.  The first operands of
// the gradient products are P and dS in tensor memory, where they replace S
// and dO V^T; the key walk computes both transposed (a lane has a key), so
// that nothing is ever transposed through shared memory.  Eight warps do the
// arithmetic, a thread half a row; one loads tiles, one issues products, one
// brings lse and delta.  The products of one half of a step run under the
// arithmetic of the other.
#include <algorithm>

#include "attn.h"
#include "launch.cuh"
#include "umma.cuh"

namespace syncgb {
namespace {

using namespace umma;

constexpr int kThreads = 384;          // 8 warps of arithmetic, 4 of which three have a role
constexpr int kRegsMany = 208, kRegsFew = 88;
static_assert(2 * kRegsMany + kRegsFew <= 3 * 168, "register split");
constexpr float kLog2e = 1.4426950408889634f;

template <int DP>
struct Layout {
  static constexpr int kTileBytes = DP / 64 * kBlockBytes;
  static constexpr int kStages = DP == 128 ? 5 : 8;         // tiles of the walk in flight
  static constexpr int kRing = 2 * kTileBytes;              // after the two tiles that stay
  static constexpr int kStats = kRing + kStages * kTileBytes;
  static constexpr int kStatStages = 2;
  static constexpr int kStatBytes = 2 * kTile * 4;          // lse, delta of a query tile
  static constexpr int kBars = kStats + kStatStages * kStatBytes;
  static constexpr int kInts = kBars + 8 * (10 + 2 * kStatStages + 2 * kStages);
  static constexpr int kBytes = kInts + 16;
};

// The barriers, each 8 bytes.
template <int DP>
struct Bars {
  using L = Layout<DP>;
  uint32_t fixed_full, fixed_free, s_full, dp_full, p_ready, ds_ready, out_full, done, stat_full, stat_free, full, free_;
  __device__ __forceinline__ explicit Bars(uint32_t at)
      : fixed_full(at), fixed_free(at + 8), s_full(at + 16), dp_full(at + 32), p_ready(at + 40), ds_ready(at + 48),
        out_full(at + 56), done(at + 64), stat_full(at + 80), stat_free(stat_full + 8 * L::kStatStages),
        full(stat_free + 8 * L::kStatStages), free_(full + 8 * L::kStages) {}
  __device__ __forceinline__ void init() const {
    bar_init(fixed_full, 1);
    bar_init(fixed_free, 1);
    bar_init(s_full, 1);
    bar_init(s_full + 8, 1);
    bar_init(dp_full, 1);
    bar_init(p_ready, 8);
    bar_init(ds_ready, 8);
    bar_init(out_full, 1);
    bar_init(done, 1);
    for (int i = 0; i < L::kStatStages; ++i) {
      bar_init(stat_full + 8 * i, 1);
      bar_init(stat_free + 8 * i, 8);
    }
    for (int i = 0; i < L::kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(free_ + 8 * i, 1);
    }
    bar_init_visible();
  }
};

// Columns [c0, c1) of this thread's lane of an accumulator, to a row of an
// output; zeros where nothing was accumulated.
template <bool BF16>
__device__ __forceinline__ void write_row(uint32_t acc, void* row, int c0, int c1, int dim, float by, bool any, bool valid) {
  const RowWriter out(row, valid);
#pragma unroll 1
  for (int c = c0; c < c1; c += 32) {
    float x[32];
    __syncwarp();
    if (any) {
      tmem_ld32(acc + c, x);
      wait_ld();
    }
    uint32_t y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = any ? pack2<BF16>(x[2 * e] * by, x[2 * e + 1] * by) : 0;
    out.write(y, 2 * c, 2 * dim);
  }
}

// Rows from `rows` on of a tile in shared memory cleared by 256 threads: they
// belong to other sequences and may hold anything, and a zero weight does not
// hide a NaN.
template <int DP>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int rows) {
  for (int b = rows * 8 + (int)threadIdx.x; b < kTile * 8; b += 256)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) *reinterpret_cast<uint4*>(tile + c * kBlockBytes + b * 16) = make_uint4(0, 0, 0, 0);
  fence_async();
}

// Loads of one block, by one warp: a ring of tiles, two tiles that stay for an item.
template <int DP>
struct Loader {
  using L = Layout<DP>;
  uint32_t base;
  const Bars<DP>& b;
  int* error;
  bool leader;
  uint32_t pos = 0, fixed = 0;
  __device__ __forceinline__ void tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) tma_load(dst + c * kBlockBytes, map, bar, 64 * c, head, row);
  }
  __device__ __forceinline__ bool stay(const CUtensorMap* m0, const CUtensorMap* m1, int head, int row) {
    if (fixed && !bar_wait(b.fixed_free, (fixed - 1) & 1, error)) return false;
    if (leader) {
      bar_expect(b.fixed_full, 2 * L::kTileBytes);
      tile(base, m0, b.fixed_full, head, row);
      tile(base + L::kTileBytes, m1, b.fixed_full, head, row);
    }
    ++fixed;
    return true;
  }
  __device__ __forceinline__ bool next(const CUtensorMap* map, int head, int row) {
    const uint32_t st = pos % L::kStages;
    if (pos >= L::kStages && !bar_wait(b.free_ + 8 * st, (pos / L::kStages - 1) & 1, error)) return false;
    if (leader) {
      bar_expect(b.full + 8 * st, L::kTileBytes);
      tile(base + L::kRing + st * L::kTileBytes, map, b.full + 8 * st, head, row);
    }
    ++pos;
    return true;
  }
  __device__ __forceinline__ void finish() {                // nothing is in flight when the block ends
#pragma unroll 1
    for (uint32_t i = pos > L::kStages ? pos - L::kStages : 0; i < pos; ++i)
      bar_wait(b.full + 8 * (i % L::kStages), i / L::kStages & 1, error);
    if (fixed) bar_wait(b.fixed_full, (fixed - 1) & 1, error);
  }
};

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dkv(const __grid_constant__ AttnArgs a,
                                                          const __grid_constant__ CUtensorMap q_map,
                                                          const __grid_constant__ CUtensorMap k_map,
                                                          const __grid_constant__ CUtensorMap v_map,
                                                          const __grid_constant__ CUtensorMap do_map) {
  using L = Layout<DP>;
  constexpr uint32_t kS = 0, kDp = 128, kDv = 256, kDk = 384;
  extern __shared__ __align__(1024) uint8_t sm[];
  const uint32_t base = smem_addr(sm);
  const Bars<DP> b(base + L::kBars);
  int* const shared_int = reinterpret_cast<int*>(sm + L::kInts);
  const int warp = uniform(threadIdx.x / 32);
  if (!swizzle_aligned(base, a.error)) return;
  if (threadIdx.x == 0) {
    b.init();
  }
  if (warp == 9) tmem_alloc<512>(smem_addr(shared_int));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[0];
  const int group = a.heads / a.kv_heads;
  const int i0 = uniform(a.k_first[blockIdx.x]), i1 = uniform(a.k_first[blockIdx.x + 1]);

  if (warp >= 8) {
    regs_down<kRegsFew>();
    const bool leader = elect_one();
    if (warp == 8) {                                        // ---- loads
      Loader<DP> load{base, b, a.error, leader};
      bool ok = true;
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.k_tile[i];
        const int n = uniform(it.n), head = uniform(it.head);
        if (!n) continue;
        ok = load.stay(&k_map, &v_map, head, (int)it.k_row);
#pragma unroll 1
        for (int h = head * group; ok && h < (head + 1) * group; ++h)
#pragma unroll 1
          for (int t = 0; ok && t < n; ++t)
            ok = load.next(&q_map, h, (int)it.q_row + t * kTile) && load.next(&do_map, h, (int)it.q_row + t * kTile);
      }
      load.finish();
    } else if (warp == 9) {                                 // ---- products
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t i_s = instr(BF16, kTile, false), i_o = instr(BF16, ksteps * 16, true);
      uint32_t pos = 0, fixed = 0, n = 0;                    // n: steps so far
      auto tile = [&](uint32_t at) { return tile_desc(base + L::kRing + at % L::kStages * L::kTileBytes); };
      auto arrived = [&](uint32_t at) { return bar_wait(b.full + 8 * (at % L::kStages), at / L::kStages & 1, a.error); };
      auto done_with = [&](uint32_t bar) {
        if (leader) commit(bar);
      };
      auto release = [&](uint32_t at) { done_with(b.free_ + 8 * (at % L::kStages)); };
      auto across = [&](uint32_t d, uint32_t x, uint32_t at) {       // keys by queries
        const uint32_t y = tile(at);
        if (leader) mma_along(tmem + d, x, y, i_s, ksteps);
      };
      auto gradient = [&](uint32_t d, uint32_t x, uint32_t at, bool add) {
        const uint32_t y = tile(at);
        if (leader) {
          mma_rows(tmem + d, tmem + x, y, i_o, add);
          mma_rows(tmem + d, tmem + x + 64, y + step_rows(4), i_o, true);
        }
      };
      const uint32_t K = tile_desc(base), V = tile_desc(base + L::kTileBytes);
      auto run = [&](int steps) {
        if (!bar_wait(b.fixed_full, fixed++ & 1, a.error) || !arrived(pos)) return false;
        fence_after();
        across(kS, K, pos);
        done_with(b.s_full);
        if (!arrived(pos + 1)) return false;
        across(kDp, V, pos + 1);
        done_with(b.dp_full);
        if (steps == 1) done_with(b.fixed_free);
#pragma unroll 1
        for (int j = 0; j < steps; ++j, pos += 2, ++n) {
          if (!bar_wait(b.p_ready, n & 1, a.error)) return false;
          fence_after();
          gradient(kDv, kS, pos + 1, j > 0);
          release(pos + 1);
          if (j + 1 < steps) {
            if (!arrived(pos + 2)) return false;
            across(kS, K, pos + 2);
            done_with(b.s_full);
          }
          if (!bar_wait(b.ds_ready, n & 1, a.error)) return false;
          fence_after();
          gradient(kDk, kDp, pos, j > 0);
          release(pos);
          if (j + 1 < steps) {
            if (!arrived(pos + 3)) return false;
            across(kDp, V, pos + 3);
            done_with(b.dp_full);
            if (j + 2 == steps) done_with(b.fixed_free);
          }
        }
        done_with(b.out_full);
        return true;
      };
#pragma unroll 1
      for (int i = i0; i < i1; ++i) {
        const int steps = uniform(a.k_tile[i].n) * group;
        if (steps && !run(steps)) break;
      }
      done_with(b.done);
      bar_wait(b.done, 0, a.error);
    } else if (warp == 10) {                                // ---- lse and delta of the query tiles
      const int lane = threadIdx.x % 32;
      uint32_t n = 0;
      bool ok = true;
      after_previous();                                      // delta is there
      let_next_start();
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.k_tile[i];
        const int tiles = uniform(it.n), head = uniform(it.head);
#pragma unroll 1
        for (int h = head * group; ok && h < (head + 1) * group; ++h)
#pragma unroll 1
          for (int t = 0; t < tiles; ++t, ++n) {
            const uint32_t st = n % L::kStatStages;
            float lse[4], delta[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int q = t * kTile + lane + 32 * e;
              lse[e] = q < it.rows ? __ldg(a.lse + h * a.q.rows + it.q_row + q) * kLog2e : -INFINITY;
              delta[e] = q < it.rows ? a.delta[h * a.delta_rows + it.q_row + q] : 0.f;
              if (lse[e] == -INFINITY) lse[e] = INFINITY;    // no weight for a row that sees nothing
            }
            if (n >= L::kStatStages && !(ok = bar_wait(b.stat_free + 8 * st, (n / L::kStatStages - 1) & 1, a.error))) break;
            float* at = reinterpret_cast<float*>(sm + L::kStats + st * L::kStatBytes);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              at[lane + 32 * e] = lse[e];
              at[kTile + lane + 32 * e] = delta[e];
            }
            bar_arrive_warp(b.stat_full + 8 * st, leader);
          }
      }
    }
  } else {                                                  // ---- arithmetic: a key per lane, 64 queries
    regs_up<kRegsMany>();
    const bool leader = elect_one();
    const int half = warp / 4, r = threadIdx.x % 128, c0 = 64 * half;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    const uint32_t S = tmem + lanes + kS + c0, Dp = tmem + lanes + kDp + c0;
    const float c2 = a.scale * kLog2e;
    uint32_t n = 0, pos = 0, items = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const AttnTile it = a.k_tile[i];
      if (i + 1 < i1) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.k_tile + i + 1));
      const int tiles = uniform(it.n), steps = tiles * group, queries = uniform(it.rows), first_seen = uniform(it.seen);
      bool ok = true;
      int t = 0;
#pragma unroll 1
      for (int j = 0; j < steps; ++j, ++n, pos += 2) {
        const uint32_t st = n % L::kStatStages;
        const float* stat = reinterpret_cast<const float*>(sm + L::kStats + st * L::kStatBytes) + c0;
        // queries [from, to) of this half see the key
        const int q0 = t * kTile, rows = queries - q0;
        const int from = r + 1 - first_seen - q0 - c0, to = rows - c0;
        const bool tail = rows < kTile, masked = first_seen + q0 < kTile || tail;
        t = t + 1 < tiles ? t + 1 : 0;
        float p[64];
        if (!(ok = bar_wait(b.stat_full + 8 * st, n / L::kStatStages & 1, a.error) && bar_wait(b.s_full, n & 1, a.error))) break;
        fence_after();
        tmem_ld32(S, p);
        tmem_ld32(S + 32, p + 32);
        wait_ld();
#pragma unroll
        for (int e = 0; e < 64; e += 4) {
          const float4 l = *reinterpret_cast<const float4*>(stat + e);
          p[e] = exp2_fast(fmaf(p[e], c2, -l.x));
          p[e + 1] = exp2_fast(fmaf(p[e + 1], c2, -l.y));
          p[e + 2] = exp2_fast(fmaf(p[e + 2], c2, -l.z));
          p[e + 3] = exp2_fast(fmaf(p[e + 3], c2, -l.w));
        }
        if (masked)
#pragma unroll
          for (int e = 0; e < 64; ++e) p[e] = e >= from && e < to ? p[e] : 0.f;
        {
          uint32_t y[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) y[e] = pack2<BF16>(p[2 * e], p[2 * e + 1]);
          tmem_st32(S, y);
        }
        if (tail) {
          const uint32_t at = pos + 1, sg = at % L::kStages;
          if (!(ok = bar_wait(b.full + 8 * sg, at / L::kStages & 1, a.error))) break;
          clear_rows<DP>(sm + L::kRing + sg * L::kTileBytes, rows);
        }
        wait_st();
        fence_before();
        bar_arrive_warp(b.p_ready, leader);
        if (!(ok = bar_wait(b.dp_full, n & 1, a.error))) break;
        fence_after();
        float d[64];
        tmem_ld32(Dp, d);
        tmem_ld32(Dp + 32, d + 32);
        wait_ld();
#pragma unroll
        for (int e = 0; e < 64; e += 4) {
          const float4 l = *reinterpret_cast<const float4*>(stat + kTile + e);
          d[e] = p[e] * (d[e] - l.x);
          d[e + 1] = p[e + 1] * (d[e + 1] - l.y);
          d[e + 2] = p[e + 2] * (d[e + 2] - l.z);
          d[e + 3] = p[e + 3] * (d[e + 3] - l.w);
        }
        if (masked)
#pragma unroll
          for (int e = 0; e < 64; ++e) d[e] = e >= from && e < to ? d[e] : 0.f;
        {
          uint32_t y[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) y[e] = pack2<BF16>(d[2 * e], d[2 * e + 1]);
          tmem_st32(Dp, y);
        }
        if (tail) clear_rows<DP>(sm + L::kRing + pos % L::kStages * L::kTileBytes, rows);   // there since S is
        wait_st();
        fence_before();
        bar_arrive_warp(b.ds_ready, leader);
        bar_arrive_warp(b.stat_free + 8 * st, leader);
      }
      if (!ok) break;
      if (steps) {
        if (!bar_wait(b.out_full, items++ & 1, a.error)) break;
        fence_after();
      }
      const AttnTensor& out = half ? a.dk : a.dv;
      uint8_t* row = static_cast<uint8_t*>(out.data) + 2 * ((it.k_row + r) * out.row + it.head * out.head);
      write_row<BF16>(tmem + lanes + (half ? kDk : kDv), row, 0, DP, a.dim, half ? a.scale : 1.f, steps > 0, r < it.keys);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 9) tmem_free<512>(tmem);
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) k_attn_dq(const __grid_constant__ AttnArgs a,
                                                         const __grid_constant__ CUtensorMap q_map,
                                                         const __grid_constant__ CUtensorMap k_map,
                                                         const __grid_constant__ CUtensorMap v_map,
                                                         const __grid_constant__ CUtensorMap do_map) {
  using L = Layout<DP>;
  constexpr uint32_t kS = 0, kDp = 256, kDq = 384;          // two buffers of scores
  extern __shared__ __align__(1024) uint8_t sm[];
  const uint32_t base = smem_addr(sm);
  const Bars<DP> b(base + L::kBars);
  int* const shared_int = reinterpret_cast<int*>(sm + L::kInts);
  const int warp = uniform(threadIdx.x / 32);
  if (!swizzle_aligned(base, a.error)) return;
  if (threadIdx.x == 0) {
    b.init();
  }
  if (warp == 9) tmem_alloc<512>(smem_addr(shared_int));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[0];
  const int group = a.heads / a.kv_heads;
  const int i0 = uniform(a.q_first[blockIdx.x]), i1 = uniform(a.q_first[blockIdx.x + 1]);

  if (warp >= 8) {
    regs_down<kRegsFew>();
    const bool leader = elect_one();
    if (warp == 8) {                                        // ---- loads
      Loader<DP> load{base, b, a.error, leader};
      bool ok = true;
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.q_tile[i];
        const int n = uniform(it.n);
        if (!n) continue;
        ok = load.stay(&q_map, &do_map, it.head, (int)it.q_row);
#pragma unroll 1
        for (int j = 0; ok && j < n; ++j)
          ok = load.next(&k_map, it.head / group, (int)it.k_row + j * kTile) &&
               load.next(&v_map, it.head / group, (int)it.k_row + j * kTile);
      }
      load.finish();
    } else if (warp == 9) {                                 // ---- products
      const int ksteps = (a.dim + 15) / 16;
      const uint32_t i_s = instr(BF16, kTile, false), i_o = instr(BF16, ksteps * 16, true);
      uint32_t pos = 0, fixed = 0, n = 0;
      auto tile = [&](uint32_t at) { return tile_desc(base + L::kRing + at % L::kStages * L::kTileBytes); };
      auto arrived = [&](uint32_t at) { return bar_wait(b.full + 8 * (at % L::kStages), at / L::kStages & 1, a.error); };
      auto done_with = [&](uint32_t bar) {
        if (leader) commit(bar);
      };
      auto release = [&](uint32_t at) { done_with(b.free_ + 8 * (at % L::kStages)); };
      const uint32_t Q = tile_desc(base), dO = tile_desc(base + L::kTileBytes);
      auto across = [&](uint32_t d, uint32_t x, uint32_t at) {       // queries by keys
        const uint32_t y = tile(at);
        if (leader) mma_along(tmem + d, x, y, i_s, ksteps);
      };
      auto scores = [&](uint32_t step, uint32_t at) {
        across(kS + step % 2 * 128, Q, at);
        done_with(b.s_full + 8 * (step % 2));
      };
      auto run = [&](int steps) {
        if (!bar_wait(b.fixed_full, fixed++ & 1, a.error) || !arrived(pos)) return false;
        fence_after();
        scores(n, pos);
        if (!arrived(pos + 1)) return false;
        across(kDp, dO, pos + 1);
        done_with(b.dp_full);
        release(pos + 1);
        if (steps > 1) {
          if (!arrived(pos + 2)) return false;
          scores(n + 1, pos + 2);
        } else {
          done_with(b.fixed_free);
        }
#pragma unroll 1
        for (int j = 0; j < steps; ++j, pos += 2, ++n) {
          if (!bar_wait(b.ds_ready, n & 1, a.error)) return false;
          fence_after();
          const uint32_t k = tile(pos);
          if (leader) {
            mma_rows(tmem + kDq, tmem + kDp, k, i_o, j > 0);
            mma_rows(tmem + kDq, tmem + kDp + 64, k + step_rows(4), i_o, true);
          }
          release(pos);
          if (j + 1 < steps) {
            if (!arrived(pos + 3)) return false;
            across(kDp, dO, pos + 3);
            done_with(b.dp_full);
            release(pos + 3);
          }
          if (j + 2 < steps) {
            if (!arrived(pos + 4)) return false;
            scores(n + 2, pos + 4);
          }
          if (j + 2 == steps) done_with(b.fixed_free);
        }
        done_with(b.out_full);
        return true;
      };
#pragma unroll 1
      for (int i = i0; i < i1; ++i) {
        const int steps = uniform(a.q_tile[i].n);
        if (steps && !run(steps)) break;
      }
      done_with(b.done);
      bar_wait(b.done, 0, a.error);
    }
  } else {                                                  // ---- arithmetic: a query per lane, 64 keys
    regs_up<kRegsMany>();
    const bool leader = elect_one();
    const int half = warp / 4, r = threadIdx.x % 128, c0 = 64 * half;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16, Dp = tmem + lanes + kDp + c0;
    const float c2 = a.scale * kLog2e;
    uint32_t n = 0, pos = 0, items = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const AttnTile it = a.q_tile[i];
      if (i + 1 < i1) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.q_tile + i + 1));
      const int steps = uniform(it.n), first_seen = uniform(it.seen), keys = uniform(it.keys);
      const int64_t query = it.q_row + r;
      const bool valid = r < it.rows;
      float lse = INFINITY, delta = 0.f;
      if (valid) {
        lse = __ldg(a.lse + it.head * a.q.rows + query) * kLog2e;
        delta = a.delta[it.head * a.delta_rows + query];
        if (lse == -INFINITY) lse = INFINITY;                // no weight for a row that sees nothing
      }
      bool ok = true;
#pragma unroll 1
      for (int j = 0; j < steps; ++j, ++n, pos += 2) {
        const uint32_t S = tmem + lanes + kS + n % 2 * 128 + c0;
        const int seen = first_seen + r - j * kTile - c0;                   // keys of this half that the row sees
        const bool masked = (j + 1) * kTile > first_seen;
        float p[64];
        if (!(ok = bar_wait(b.s_full + 8 * (n % 2), n / 2 & 1, a.error))) break;
        fence_after();
        tmem_ld32(S, p);
        tmem_ld32(S + 32, p + 32);
        wait_ld();
#pragma unroll
        for (int e = 0; e < 64; ++e) p[e] = exp2_fast(fmaf(p[e], c2, -lse));
        if (!(ok = bar_wait(b.dp_full, n & 1, a.error))) break;
        fence_after();
        float d[64];
        tmem_ld32(Dp, d);
        tmem_ld32(Dp + 32, d + 32);
        wait_ld();
#pragma unroll
        for (int e = 0; e < 64; ++e) d[e] = p[e] * (d[e] - delta);
        if (masked)
#pragma unroll
          for (int e = 0; e < 64; ++e) d[e] = e < seen ? d[e] : 0.f;
        {
          uint32_t y[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) y[e] = pack2<BF16>(d[2 * e], d[2 * e + 1]);
          tmem_st32(Dp, y);
        }
        if ((j + 1) * kTile > keys) clear_rows<DP>(sm + L::kRing + pos % L::kStages * L::kTileBytes, keys - j * kTile);
        wait_st();
        fence_before();
        bar_arrive_warp(b.ds_ready, leader);
      }
      if (!ok) break;
      if (steps) {
        if (!bar_wait(b.out_full, items++ & 1, a.error)) break;
        fence_after();
      }
      uint8_t* row = static_cast<uint8_t*>(a.dq.data) + 2 * (query * a.dq.row + it.head * a.dq.head);
      write_row<BF16>(tmem + lanes + kDq, row, half * DP / 2, (half + 1) * DP / 2, a.dim, a.scale, steps > 0, valid);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 9) tmem_free<512>(tmem);
  after_previous();                                          // no later kernel overtakes the key walk
}

// delta of every row and head, eight entries per lane; LANES lanes a head.
template <int LANES, bool BF16>
__global__ void __launch_bounds__(256) k_attn_delta(const __grid_constant__ AttnArgs a) {
  let_next_start();
  const int64_t unit = (blockIdx.x * 256ll + threadIdx.x) / LANES;
  const int e = threadIdx.x % LANES * 8;
  const int64_t row = unit / a.heads;
  const int head = (int)(unit - row * a.heads);
  float sum = 0.f;
  if (row < a.delta_rows && e < a.dim) {
    const uint8_t *o = static_cast<const uint8_t*>(a.o.data), *g = static_cast<const uint8_t*>(a.d_o.data);
    const uint4 x = *reinterpret_cast<const uint4*>(o + 2 * (row * a.o.row + head * a.o.head + e));
    const uint4 y = *reinterpret_cast<const uint4*>(g + 2 * (row * a.d_o.row + head * a.d_o.head + e));
    const uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack2<BF16>(u[i]), h = unpack2<BF16>(v[i]);
      sum = fmaf(f.x, h.x, fmaf(f.y, h.y, sum));
    }
  }
#pragma unroll
  for (int i = LANES / 2; i > 0; i >>= 1) sum += __shfl_xor_sync(~0u, sum, i);
  if (row < a.delta_rows && threadIdx.x % LANES == 0) a.delta[head * a.delta_rows + row] = sum;
}

// The walks start early: the key walk's loads and products run before delta is
// there, and the query walk, which needs nothing of the key walk, takes the
// SMs that its last blocks leave.  (The key walk's blocks let it start only
// once delta is there.)
template <class K>
cudaError_t walk(K kernel, int blocks, int bytes, std::atomic<uint64_t>& allowed, const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  cudaError_t e = allow_smem(kernel, bytes, allowed);
  if (e != cudaSuccess) return e;
  e = launch_early(kernel, blocks, kThreads, bytes, st, a, m.q, m.k, m.v, m.d_o);
  if (e == cudaSuccess) count_launch();
  return e;
}

template <int DP, bool BF16>
cudaError_t launch(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  using L = Layout<DP>;
  static_assert(L::kBytes <= 227 * 1024, "shared memory");
  static std::atomic<uint64_t> dkv_allowed{0}, dq_allowed{0};
  cudaError_t e = cudaSuccess;
  if (a.delta_rows) {
    const int64_t blocks = (a.delta_rows * a.heads * (DP / 8) + 255) / 256;
    k_attn_delta<DP / 8, BF16><<<(unsigned)blocks, 256, 0, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    count_launch();
  }
  if (a.n_k_blocks && (e = walk(k_attn_dkv<DP, BF16>, a.n_k_blocks, L::kBytes, dkv_allowed, a, m, st)) != cudaSuccess) return e;
  if (a.n_q_blocks && (e = walk(k_attn_dq<DP, BF16>, a.n_q_blocks, L::kBytes, dq_allowed, a, m, st)) != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_attn_backward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  if (a.dim <= 64) return a.bf16 ? launch<64, true>(a, m, st) : launch<64, false>(a, m, st);
  return a.bf16 ? launch<128, true>(a, m, st) : launch<128, false>(a, m, st);
}

}  // namespace syncgb

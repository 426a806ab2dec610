// Forward attention over packed sequences (include/sync.h, sync_attn_forward).
//
// One block per SM takes work items in turn: two query tiles of 128 rows
// against a range of 128-key tiles, S = Q K^T and O += P V on the tensor
// cores with accumulators in tensor memory.  Warps by role: four for the
// softmax of each query tile (a thread has a row, so its maximum and sum need
// no exchange), one that loads keys and values, one that loads queries, and
// one that issues the products of each query tile.  The two query tiles share
// the loads and go at their own pace: while one's softmax runs, the other's
// products do, also from one item to the next.  P replaces S in tensor memory
// as the first operand of the second product and never passes through shared
// memory.
//
// Rows of a tile are consecutive queries of one head, or, where a sequence
// has few queries, the queries of all heads of a group (row = query * group +
// head): their keys are then read once for the group.  A key range that would
// leave SMs idle is split into pieces, whose results a second kernel merges.
//
// Bounds.  A pair of tiles takes 1024 cycles of products (128 x 128 x 128
// twice at 4096 a cycle), which is also what shared memory takes to deliver
// their operands and to receive the next tiles (128 KB at 128 bytes a cycle),
// and 512 of exponentials.  Measured on 8192 tokens, 32 heads of 128: 370 us,
// 1490 TFLOP/s of the visible pairs (alone; 397 when passes follow one another
// and the power limit holds), 1550 cycles a pair of tiles, the tensor pipe busy
// 66% of them; the rest is the way from a tile's scores to its
// weights (700 cycles of exponentials of one row per thread, 100 for the
// scores, barriers on both sides) where the other query tile's products do
// not cover it.  Half a row per thread on twice the warps took 414 us, whole
// rows loaded from tensor memory in two passes 405.  64 decode steps on caches
// of 1 to 8096 keys, 8 key heads: 63.5 us, 5.8 TB/s while tiles stream.
#include <algorithm>

#include "attn.h"
#include "launch.cuh"
#include "umma.cuh"

namespace syncgb {
namespace {

using namespace umma;

constexpr int kThreads = 384;          // two softmax groups of 4 warps, and 4 warps with a role each
// Registers per thread: 168 at launch (3 warpgroups of 168 = 504), of which
// the softmax groups take most, so that a row of scores stays in registers.
constexpr int kRegsMany = 224, kRegsFew = 56;
static_assert(2 * kRegsMany + kRegsFew <= 3 * 168, "register split");
constexpr int kCols = 512;
// columns of query tile t's scores and outputs
__device__ __forceinline__ constexpr uint32_t s_col(int t) { return 128 * t; }
__device__ __forceinline__ constexpr uint32_t o_col(int t) { return 256 + 128 * t; }

template <int DP>
struct Layout {
  static constexpr int kTileBytes = DP / 64 * kBlockBytes;
  static constexpr int kStages = DP == 128 ? 5 : 10;        // key and value tiles in flight
  static constexpr int kRing = 2 * kTileBytes;              // after the two query tiles
  static constexpr int kBars = kRing + kStages * kTileBytes;
  static constexpr int kInts = kBars + 104 + 16 * kStages;  // after the barriers: where tensor memory is
  static constexpr int kBytes = kInts + 8;
};

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) k_attn_fwd(const __grid_constant__ AttnArgs a,
                                                          const __grid_constant__ CUtensorMap q_map,
                                                          const __grid_constant__ CUtensorMap qg_map,
                                                          const __grid_constant__ CUtensorMap k_map,
                                                          const __grid_constant__ CUtensorMap v_map) {
  using L = Layout<DP>;
  extern __shared__ __align__(1024) uint8_t sm[];
  const uint32_t base = smem_addr(sm), bars = base + L::kBars;
  const uint32_t q_full = bars, q_free = bars + 16, s_full = bars + 32, p_full = bars + 48, o_full = bars + 64,
                 p_half = bars + 80, done = bars + 96, full = bars + 104, free_ = full + 8 * L::kStages;
  int* const shared_int = reinterpret_cast<int*>(sm + L::kInts);
  const int warp = uniform(threadIdx.x / 32);
  if (!swizzle_aligned(base, a.error)) return;
  if (threadIdx.x == 0) {
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      bar_init(q_full + 8 * t, 1);
      bar_init(q_free + 8 * t, 1);
      bar_init(s_full + 8 * t, 1);
      bar_init(p_half + 8 * t, 4);
      bar_init(p_full + 8 * t, 4);
      bar_init(o_full + 8 * t, 1);
    }
    bar_init(done, 2);
#pragma unroll 1
    for (int i = 0; i < L::kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(free_ + 8 * i, 2);
    }
    bar_init_visible();
  }
  if (warp == 8) tmem_alloc<kCols>(smem_addr(shared_int));
  const int i0 = uniform(a.block_first[blockIdx.x]), i1 = uniform(a.block_first[blockIdx.x + 1]);
  asm volatile("prefetch.global.L1 [%0];" ::"l"(a.item + i0));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[0];

  const int group = a.heads / a.kv_heads, packed_rows = kTile / group;
  if (threadIdx.x == 0) let_next_start();

  if (warp >= 8) {
    regs_down<kRegsFew>();
    const bool leader = elect_one();
    if (warp == 8) {                                        // ---- loads of key and value tiles
      Place<L::kStages> at;
      bool ok = true, first = true;                         // first: of the ring, whose places are free
      auto load = [&](const CUtensorMap* map, int head, int row) {
        const uint32_t bar = full + 8 * at.stage;
        if (!first && !bar_wait(free_ + 8 * at.stage, at.parity ^ 1, a.error)) return false;
        if (leader) {
          bar_expect(bar, L::kTileBytes);
#pragma unroll
          for (int c = 0; c < DP / 64; ++c)
            tma_load(base + L::kRing + at.stage * L::kTileBytes + c * kBlockBytes, map, bar, 64 * c, head, row);
        }
        at.next();
        first = first && at.stage;
        return true;
      };
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnItem it = a.item[i];
        const int n = 2 * uniform(max(it.n[0], it.n[1])), head = it.head / group;
        int row = (int)it.k_row;
#pragma unroll 1
        for (int j = 0; ok && j < n; ++j) {                  // a key tile, then its value tile
          ok = load(j % 2 ? &v_map : &k_map, head, row);
          row += j % 2 * kTile;
        }
      }
      // nothing is in flight when the block ends
#pragma unroll 1
      for (int i = 0; i < L::kStages; ++i) {
        if (!first || (uint32_t)i < at.stage) bar_wait(full + 8 * i, at.parity ^ ((uint32_t)i >= at.stage), a.error);
      }
    } else if (warp == 9) {                                 // ---- loads of query tiles
      uint32_t n[2] = {0, 0};
      bool ok = true;
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnItem it = a.item[i];
        const int packed = uniform(it.packed), row = (int)it.q_row, apart = packed ? packed_rows : kTile;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (!ok || !uniform(it.n[t])) continue;
          if (n[t] && !(ok = bar_wait(q_free + 8 * t, (n[t] - 1) & 1, a.error))) continue;
          if (leader) {
            bar_expect(q_full + 8 * t, DP / 64 * (packed ? packed_rows * group : kTile) * 128);
#pragma unroll
            for (int c = 0; c < DP / 64; ++c)
              tma_load(base + t * L::kTileBytes + c * kBlockBytes, packed ? &qg_map : &q_map, q_full + 8 * t, 64 * c,
                       it.head, row + t * apart);
          }
          ++n[t];
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (n[t]) bar_wait(q_full + 8 * t, (n[t] - 1) & 1, a.error);
    } else {                                                // ---- products of query tile t
      const int t = warp - 10, ksteps = (a.dim + 15) / 16;
      const uint32_t i_s = instr(BF16, kTile, false), i_o = instr(BF16, ksteps * 16, true);
      const uint32_t S = tmem + s_col(t), O = tmem + o_col(t);
      const uint32_t Q = tile_desc(base + t * L::kTileBytes), ring = tile_desc(base + L::kRing);
      Place<L::kStages> at;                                  // of the next tile
      uint32_t items = 0, steps = 0;
      auto arrived = [&] { return bar_wait(full + 8 * at.stage, at.parity, a.error); };
      auto tile = [&] { return ring + at.stage * (L::kTileBytes >> 4); };
      auto scores = [&](bool first, bool last) {
        if (!arrived() || (first && !bar_wait(q_full + 8 * t, items++ & 1, a.error))) return false;
        fence_after();
        if (leader) {
          mma_along(S, Q, tile(), i_s, ksteps);
          commit(s_full + 8 * t);
          commit(free_ + 8 * at.stage);
          if (last) commit(q_free + 8 * t);
        }
        at.next();
        return true;
      };
      auto run = [&](int n, int all) {                      // the first n of the item's key tiles are this query tile's
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
          if (j == 0 && !scores(true, n == 1)) return false;
          const uint32_t v = tile(), v_free = free_ + 8 * at.stage;
          if (!arrived() || !bar_wait(p_half + 8 * t, steps & 1, a.error)) return false;
          fence_after();
          if (leader) mma_rows(O, S, v, i_o, j > 0);
          at.next();
          if (!bar_wait(p_full + 8 * t, steps++ & 1, a.error)) return false;
          fence_after();
          if (leader) {
            mma_rows(O, S + 32, v + step_rows(4), i_o, true);
            commit(v_free);
            if (j + 1 == n) commit(o_full + 8 * t);
          }
          if (j + 1 < n && !scores(false, j + 2 == n)) return false;
        }
#pragma unroll 1
        for (int j = 2 * n; j < 2 * all; ++j, at.next()) {   // the other's: let go as they come
          if (!arrived()) return false;
          bar_arrive_warp(free_ + 8 * at.stage, leader);
        }
        return true;
      };
#pragma unroll 1
      for (int i = i0; i < i1; ++i) {
        const AttnItem* const it = a.item + i;
        if (!run(uniform(it->n[t]), uniform(max(it->n[0], it->n[1])))) break;
      }
      if (leader) commit(done);
      bar_wait(done, 0, a.error);
    }
  } else {                                                  // ---- softmax: a row of query tile t per thread
    regs_up<kRegsMany>();
    const int t = warp / 4, r = threadIdx.x % 128;
    const bool leader = elect_one();
    const int packed_q = r / group, packed_h = r % group;    // query and head of a packed tile's row
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16, S = tmem + s_col(t) + lanes, O = tmem + o_col(t) + lanes;
    const float c2 = a.scale * 1.4426950408889634f;          // weights are powers of two
    const float slack = 8.f / c2;                            // see below
    uint32_t pos = 0, sn = 0, on = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const AttnItem* const at_item = a.item + i;
      if (i + 1 < i1) asm volatile("prefetch.global.L1 [%0];" ::"l"(at_item + 1));
      const int packed = uniform(at_item->packed), n = uniform(at_item->n[t]), keys = uniform(at_item->keys);
      const int per = packed ? packed_rows : kTile, rq = packed ? packed_q : r;
      const int least = uniform(at_item->seen) + t * per;   // keys that the tile's first query sees
      const int seen_all = min(least + rq, keys);            // and this row
      const bool valid = rq < at_item->rows[t], busy = __any_sync(~0u, valid);
      float m = -INFINITY, l = 0.f;
      bool ok = true;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int k0 = j * kTile;
        if (!(ok = bar_wait(s_full + 8 * t, sn++ & 1, a.error))) break;
        if (k0 + kTile > keys) {
          // Values past the sequence's end belong to other sequences and may
          // be anything; a zero weight does not hide a NaN, so they are
          // cleared (both query tiles write the same zeros).
          const uint32_t at = pos + 2 * j + 1, st = at % L::kStages;
          if (!(ok = bar_wait(full + 8 * st, at / L::kStages & 1, a.error))) break;
          uint8_t* v = sm + L::kRing + st * L::kTileBytes;
#pragma unroll 1
          for (int b = (keys - k0) * 8 + r; b < kTile * 8; b += 128)
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) *reinterpret_cast<uint4*>(v + c * kBlockBytes + b * 16) = make_uint4(0, 0, 0, 0);
          fence_async();
        }
        if (!busy) {                                         // rows that nobody asked for
          bar_arrive_warp(p_half + 8 * t, leader);
          bar_arrive_warp(p_full + 8 * t, leader);
          continue;
        }
        fence_after();
        if (k0 + kTile > least) {                             // some row does not see the whole tile
          const int seen = seen_all - k0;
#pragma unroll 1
          for (int c = max(0, uniform(seen)) & ~15; c < kTile; c += 16) keep16(S + c, 0, seen - c, -INFINITY);
          wait_st();
        }
        float x[kTile];
#pragma unroll
        for (int c = 0; c < kTile; c += 32) tmem_ld32(S + c, x + c);
        wait_ld();
        // (The weights are rounded to the operands' type, which is what the
        // second product takes; their sum is of the unrounded ones.)
        // The weights of the first half with the maximum known so far, while
        // the tile's own is found (the one keeps the special function unit
        // busy, the other the integer unit).
        const uint64_t c22 = pair_bits(c2, c2);
        uint64_t l2[2];
        uint32_t y[kTile / 4];
        auto weights = [&](const float* s, uint32_t* p) {
          const float shift = m == -INFINITY ? 0.f : m * c2;
          const uint64_t shift2 = pair_bits(-shift, -shift);
#pragma unroll
          for (int e = 0; e < kTile / 2; e += 2) {
            float u, v;
            pair_split(fma2(pair_bits(s[e], s[e + 1]), c22, shift2), u, v);
            u = exp2_fast(u);
            v = exp2_fast(v);
            l2[e / 2 % 2] = add2(l2[e / 2 % 2], pair_bits(u, v));
            p[e / 2] = pack2<BF16>(u, v);
          }
        };
        l2[0] = l2[1] = 0;
        weights(x, y);
        float m4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int c = 4; c < kTile; c += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) m4[e] = fmaxf(m4[e], c + 4 + e < kTile ? fmaxf(x[c + e], x[c + 4 + e]) : x[c + e]);
        const float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
        // The running maximum follows only rises of more than 2^8 in the
        // weights: until then they may grow to 2^8, which neither 16-bit type
        // nor the 32-bit sums mind, and O needs no new scale.  Every row
        // decides for itself, so that no other row of its tile changes its
        // rounding.  All products up to the last tile's are done when this
        // tile's scores are.
        const bool rises = j == 0 || top > m + slack;
        if (__any_sync(~0u, rises)) {
          const float by = rises && j > 0 ? exp2_fast((m - top) * c2) : 1.f;
          m = rises ? top : m;
          l *= by;
          if (j > 0)
#pragma unroll 1
            for (int c = 0; c < DP; c += 16) {
              float o[16];
              tmem_ld16(O + c, o);
              wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] *= by;
              tmem_st16(O + c, reinterpret_cast<uint32_t*>(o));
            }
          l2[0] = l2[1] = 0;
          weights(x, y);
        }
        tmem_st32(S, y);
        wait_st();                                            // the first half may be multiplied
        fence_before();
        bar_arrive_warp(p_half + 8 * t, leader);
        weights(x + kTile / 2, y);
        tmem_st32(S + 32, y);
        wait_st();
        fence_before();
        bar_arrive_warp(p_full + 8 * t, leader);
        float l4[4];
        pair_split(l2[0], l4[0], l4[1]);
        pair_split(l2[1], l4[2], l4[3]);
        l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
      }
      if (!ok) break;
      pos += 2 * uniform(max(at_item->n[0], at_item->n[1]));
      if (n) {
        if (!bar_wait(o_full + 8 * t, on++ & 1, a.error)) break;
        fence_after();
      }
      if (!busy) continue;
      const bool some = n && l != 0.f;
      const float by = __fdividef(1.f, l);
      const int slot = uniform(at_item->slot);
      const int head = at_item->head + (packed ? packed_h : 0);
      const int64_t query = at_item->q_row + t * per + rq;
      if (valid) {
        const float lse2 = l == 0.f ? -INFINITY : fmaf(m, c2, __log2f(l));
        if (slot >= 0)
          a.part_lse[((int64_t)slot * 2 + t) * kTile + r] = lse2;
        else if (a.lse)
          a.lse[head * a.q.rows + query] = lse2 * 0.6931471805599453f;
      }
      // A piece of a split key range leaves its rows in 32 bits, scaled by its
      // own sum; whole ranges are done.
      const bool piece = slot >= 0;
      const RowWriter out(piece ? reinterpret_cast<uint8_t*>(a.part_o + (((int64_t)slot * 2 + t) * kTile + r) * DP)
                                : static_cast<uint8_t*>(a.o.data) + 2 * (query * a.o.row + head * a.o.head),
                          valid);
#pragma unroll 1
      for (int c = 0; c < DP; c += piece ? 16 : 32) {
        float o[32];
        uint32_t y[16];
        __syncwarp();
        tmem_ld32(O + min(c, DP - 32), o);
        wait_ld();
        if (piece) {                                         // (the last 16 columns come in the upper half)
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = some ? __float_as_uint(o[c > DP - 32 ? e + 16 : e] * by) : 0;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = some ? pack2<BF16>(o[2 * e] * by, o[2 * e + 1] * by) : 0;
        }
        out.write(y, piece ? 4 * c : 2 * c, piece ? 4 * DP : 2 * a.dim);
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 8) tmem_free<kCols>(tmem);
}

// Rows of split key ranges from their pieces, in the order of the pieces: a
// warp per row, four columns per lane (of the first DP / 4 lanes).
template <int DP, bool BF16>
__global__ void __launch_bounds__(256) k_attn_merge(const __grid_constant__ AttnArgs a) {
  after_previous();
  const AttnSplit s = a.split[blockIdx.x];
  const int group = a.heads / a.kv_heads, heads = s.packed ? group : 1, lane = threadIdx.x % 32;
  int row = blockIdx.y * 8 + threadIdx.x / 32;
  const int n0 = s.rows[0] * heads, t = row >= n0;
  if (t) row -= n0;
  if (row >= s.rows[t] * heads) return;
  const float* lse = a.part_lse + ((int64_t)s.slot * 2 + t) * kTile + row;
  const float* part = a.part_o + (((int64_t)s.slot * 2 + t) * kTile + row) * DP + lane % (DP / 4) * 4;
  float top = -INFINITY;
  for (int k = lane; k < s.pieces; k += 32) top = fmaxf(top, lse[(int64_t)k * 2 * kTile]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  const float from = top == -INFINITY ? 0.f : top;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int k = 0; k < s.pieces; ++k) {
    const float f = exp2_fast(lse[(int64_t)k * 2 * kTile] - from);
    const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)k * 2 * kTile * DP);
    sum += f;
    acc.x = fmaf(f, x.x, acc.x);
    acc.y = fmaf(f, x.y, acc.y);
    acc.z = fmaf(f, x.z, acc.z);
    acc.w = fmaf(f, x.w, acc.w);
  }
  const float by = sum == 0.f ? 0.f : 1.f / sum;
  const int head = s.packed ? s.head + row % group : s.head;
  const int64_t query = s.q_row + t * (s.packed ? kTile / group : kTile) + (s.packed ? row / group : row);
  if (lane < DP / 4 && lane * 4 < a.dim) {
    uint2 v;
    v.x = pack2<BF16>(acc.x * by, acc.y * by);
    v.y = pack2<BF16>(acc.z * by, acc.w * by);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.o.data) + 2 * (query * a.o.row + head * a.o.head + lane * 4)) = v;
  }
  if (a.lse && lane == 0) a.lse[head * a.q.rows + query] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

// For tests: a wait for a barrier that nobody arrives on, by the first of two
// warps, and one by the second for the first's arrival, which then never comes.
__global__ void __launch_bounds__(64) k_wait_in_vain(int* error, int tries) {
  __shared__ __align__(8) uint64_t bars[2];
  const uint32_t bar = smem_addr(bars);
  const int warp = uniform(threadIdx.x / 32);
  if (threadIdx.x == 0) {
    bar_init(bar, 1);
    bar_init(bar + 8, 1);
    bar_init_visible();
  }
  __syncthreads();
  if (bar_wait(bar + 8 * warp, 0, error, tries) && warp == 0) bar_arrive_warp(bar + 8, elect_one());
  __syncthreads();
}

template <int DP, bool BF16>
cudaError_t launch(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  using L = Layout<DP>;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(k_attn_fwd<DP, BF16>, L::kBytes, allowed);
  if (e != cudaSuccess) return e;
  k_attn_fwd<DP, BF16><<<a.n_blocks, kThreads, L::kBytes, st>>>(a, m.q, m.q_group, m.k, m.v);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  count_launch();
  if (!a.n_splits) return cudaSuccess;
  const dim3 grid((unsigned)a.n_splits, (unsigned)(a.merge_rows + 7) / 8);
  if ((e = launch_early(k_attn_merge<DP, BF16>, grid, 256, 0, st, a)) == cudaSuccess) count_launch();
  return e;
}

}  // namespace

cudaError_t launch_wait_in_vain(int* error, int tries, cudaStream_t st) {
  k_wait_in_vain<<<1, 64, 0, st>>>(error, std::min(tries, kTries));
  return cudaGetLastError();
}

cudaError_t launch_attn_forward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  if (a.dim <= 64) return a.bf16 ? launch<64, true>(a, m, st) : launch<64, false>(a, m, st);
  return a.bf16 ? launch<128, true>(a, m, st) : launch<128, false>(a, m, st);
}

}  // namespace syncgb

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
// Products read shared memory at 128 bytes a cycle at most: 8 KB for a step of
// 128 x 128 x 16 with both operands there, as long as the step takes.  So the
// query walk keeps Q and dO, first operands that stay for an item, in tensor
// memory (8192 tokens, 32 heads of 128: 623 -> 490 us, 2100 cycles a pair of
// tiles of which the products take 1536).  The key walk has no room there
// beside two accumulators: 620 us, 2700 cycles, of which products and
// shared memory take 2048 each.
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
  uint32_t fixed_full, fixed_free, s_full, fixed_ready, dp_full, p_ready, ds_ready, out_full, done, stat_full, stat_free, full, free_;
  __device__ __forceinline__ explicit Bars(uint32_t at)
      : fixed_full(at), fixed_free(at + 8), s_full(at + 16), fixed_ready(at + 24), dp_full(at + 32), p_ready(at + 40), ds_ready(at + 48),
        out_full(at + 56), done(at + 64), stat_full(at + 80), stat_free(stat_full + 8 * L::kStatStages),
        full(stat_free + 8 * L::kStatStages), free_(full + 8 * L::kStages) {}
  // fixed_users: arrivals that free the two tiles that stay
  __device__ __forceinline__ void init(int fixed_users) const {
    bar_init(fixed_full, 1);
    bar_init(fixed_free, fixed_users);
    bar_init(fixed_ready, 8);
    bar_init(s_full, 1);
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
    tmem_ld32(acc + c, x);
    wait_ld();
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
  Place<L::kStages> at;
  bool first = true;             // of the ring, whose places are free
  uint32_t fixed = 0;
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
  // n rows of tiles from `row` on, of two tensors in turn
  __device__ __forceinline__ bool pairs(const CUtensorMap* m0, const CUtensorMap* m1, int head, int row, int n) {
#pragma unroll 1
    for (int j = 0; j < 2 * n; ++j) {
      if (!first && !bar_wait(b.free_ + 8 * at.stage, at.parity ^ 1, error)) return false;
      const uint32_t bar = b.full + 8 * at.stage;
      if (leader) {
        bar_expect(bar, L::kTileBytes);
        tile(base + L::kRing + at.stage * L::kTileBytes, j % 2 ? m1 : m0, bar, head, row + j / 2 * kTile);
      }
      at.next();
      first = first && at.stage;
    }
    return true;
  }
  __device__ __forceinline__ void finish() {                // nothing is in flight when the block ends
#pragma unroll 1
    for (uint32_t i = 0; i < L::kStages; ++i)
      if (!first || i < at.stage) bar_wait(b.full + 8 * i, at.parity ^ (i >= at.stage), error);
    if (fixed) bar_wait(b.fixed_full, (fixed - 1) & 1, error);
  }
};

// Products of one block, by one warp, in the order of its ring of tiles.
template <int DP, bool BF16>
struct Products {
  using L = Layout<DP>;
  uint32_t ring, tmem;
  const Bars<DP>& b;
  int* error;
  bool leader;
  int ksteps;
  uint32_t i_s, i_o;
  Place<L::kStages> at;          // of the next tile
  __device__ __forceinline__ Products(uint32_t base, uint32_t tmem, const Bars<DP>& b, int* error, int dim)
      : ring(tile_desc(base + L::kRing)), tmem(tmem), b(b), error(error), leader(elect_one()), ksteps((dim + 15) / 16),
        i_s(instr(BF16, kTile, false)), i_o(instr(BF16, ksteps * 16, true)) {}
  __device__ __forceinline__ uint32_t tile(uint32_t stage) const { return ring + stage * (L::kTileBytes >> 4); }
  __device__ __forceinline__ void done_with(uint32_t bar) const {
    if (leader) commit(bar);
  }
  __device__ __forceinline__ void release(uint32_t stage) const { done_with(b.free_ + 8 * stage); }
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t n) const {
    const bool ok = bar_wait(bar, n & 1, error);
    fence_after();
    return ok;
  }
  // d = x y^T with the next tile y, whose stage it returns; x a tile in shared
  // memory or (TMEM) in tensor memory
  template <bool TMEM>
  __device__ __forceinline__ bool across(uint32_t d, uint32_t x, uint32_t bar, uint32_t& stage) {
    if (!wait(b.full + 8 * at.stage, at.parity)) return false;
    stage = at.stage;
    if (leader) {
      if (TMEM)
        mma_tmem_along(tmem + d, tmem + x, tile(stage), i_s, ksteps);
      else
        mma_along(tmem + d, x, tile(stage), i_s, ksteps);
      commit(bar);
    }
    at.next();
    return true;
  }
  // d (+)= x y with x of 128 columns in two runs of 64, each in its first 32 words
  __device__ __forceinline__ void gradient(uint32_t d, uint32_t x, uint32_t stage, bool add) const {
    if (!leader) return;
#pragma unroll 1
    for (int e = 0; e < 2; ++e) mma_rows(tmem + d, tmem + x + 64 * e, tile(stage) + step_rows(4 * e), i_o, add || e);
  }
};

// Weights of 64 scores, exp2(s c2 - lse2), in place, with lse2 negated: one
// value, or one for each column.
__device__ __forceinline__ void weights(float* p, float c2, const float* minus_lse, bool by_column) {
  const uint64_t c22 = pair_bits(c2, c2), all = pair_bits(*minus_lse, *minus_lse);
#pragma unroll
  for (int e = 0; e < 64; e += 4) {
    ulonglong2 l = make_ulonglong2(all, all);
    if (by_column) l = *reinterpret_cast<const ulonglong2*>(minus_lse + e);
    pair_split(fma2(pair_bits(p[e], p[e + 1]), c22, l.x), p[e], p[e + 1]);
    pair_split(fma2(pair_bits(p[e + 2], p[e + 3]), c22, l.y), p[e + 2], p[e + 3]);
#pragma unroll
    for (int f = 0; f < 4; ++f) p[e + f] = exp2_fast(p[e + f]);
  }
}
// Their gradients p (d - delta), into d, with delta negated.
__device__ __forceinline__ void weight_gradients(float* d, const float* p, const float* minus_delta, bool by_column) {
  const uint64_t all = pair_bits(*minus_delta, *minus_delta);
#pragma unroll
  for (int e = 0; e < 64; e += 4) {
    ulonglong2 l = make_ulonglong2(all, all);
    if (by_column) l = *reinterpret_cast<const ulonglong2*>(minus_delta + e);
    pair_split(mul2(pair_bits(p[e], p[e + 1]), add2(pair_bits(d[e], d[e + 1]), l.x)), d[e], d[e + 1]);
    pair_split(mul2(pair_bits(p[e + 2], p[e + 3]), add2(pair_bits(d[e + 2], d[e + 3]), l.y)), d[e + 2], d[e + 3]);
  }
}
// 64 values rounded to 16 bits, to tensor memory: P and dS, each rounded once as
// an operand of the next product.  float16 holds dS in steps of 2^-24 at the
// least and up to 65504; the caller scales d_o (include/sync.h).
template <bool BF16>
__device__ __forceinline__ void put(uint32_t addr, const float* x) {
  uint32_t y[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) y[e] = pack2<BF16>(x[2 * e], x[2 * e + 1]);
  tmem_st32(addr, y);
}
// A row of a tile in shared memory, to tensor memory as a first operand.
template <int DP>
__device__ __forceinline__ void tile_to_tmem(uint32_t addr, const uint8_t* tile, int row) {
#pragma unroll 1
  for (int c = 0; c < DP / 64; ++c) {
    uint4 x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)                              // 16-byte pieces lie at their number xor the row's
      x[e] = *reinterpret_cast<const uint4*>(tile + c * kBlockBytes + row * 128 + (e ^ row % 8) * 16);
    tmem_st32(addr + 32 * c, reinterpret_cast<const uint32_t*>(x));
  }
  wait_st();
}
__device__ __forceinline__ void get(uint32_t addr, float* x) {
  tmem_ld32(addr, x);
  tmem_ld32(addr + 32, x + 32);
  wait_ld();
}

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
  if (threadIdx.x == 0) b.init(1);
  if (warp == 9) tmem_alloc<512>(smem_addr(shared_int));
  const int group = a.heads / a.kv_heads;
  const int i0 = uniform(a.k_first[blockIdx.x]), i1 = uniform(a.k_first[blockIdx.x + 1]);
  asm volatile("prefetch.global.L1 [%0];" ::"l"(a.k_tile + i0));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[0];

  if (warp >= 8) {
    regs_down<kRegsFew>();
    if (warp == 8) {                                        // ---- loads
      Loader<DP> load{base, b, a.error, elect_one()};
      bool ok = true;
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.k_tile[i];
        const int n = uniform(it.n), head = uniform(it.head);
        if (!n) continue;
        ok = load.stay(&k_map, &v_map, head, (int)it.k_row);
#pragma unroll 1
        for (int h = head * group; ok && h < (head + 1) * group; ++h) ok = load.pairs(&q_map, &do_map, h, (int)it.q_row, n);
      }
      load.finish();
    } else if (warp == 9) {                                 // ---- products
      Products<DP, BF16> m(base, tmem, b, a.error, a.dim);
      const uint32_t K = tile_desc(base), V = tile_desc(base + L::kTileBytes);
      uint32_t fixed = 0, n = 0;                            // n: steps so far
      // The scores and dO V^T of step j + 1 each follow the gradient product
      // of step j that reads what they overwrite.
      auto run = [&](int steps) {
        uint32_t q[2], g[2];                                // stages of Q and dO of this step and the next
#pragma unroll 1
        for (int j = -1; j < steps; ++j) {
          const bool more = j + 1 < steps;
          if (j < 0) {
            if (!m.wait(b.fixed_full, fixed++)) return false;
          } else {
            if (!m.wait(b.p_ready, n)) return false;
            m.gradient(kDv, kS, g[0], j > 0);
            m.release(g[0]);
          }
          if (more && !m.template across<false>(kS, K, b.s_full, q[1])) return false;
          if (j >= 0) {
            if (!m.wait(b.ds_ready, n++)) return false;
            m.gradient(kDk, kDp, q[0], j > 0);
            m.release(q[0]);
          }
          if (more && !m.template across<false>(kDp, V, b.dp_full, g[1])) return false;
          if (j + 2 == steps) m.done_with(b.fixed_free);
          q[0] = q[1];
          g[0] = g[1];
        }
        m.done_with(b.out_full);
        return true;
      };
#pragma unroll 1
      for (int i = i0; i < i1; ++i) {
        const int steps = uniform(a.k_tile[i].n) * group;
        if (steps && !run(steps)) break;
      }
      m.done_with(b.done);
      bar_wait(b.done, 0, a.error);
    } else if (warp == 10) {                                // ---- lse and delta of the query tiles, negated
      const int lane = threadIdx.x % 32;
      const bool leader = elect_one();
      Place<L::kStatStages> at;
      bool ok = true, first = true;
      after_previous();                                      // delta is there
      let_next_start();
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.k_tile[i];
        const int tiles = uniform(it.n), head = uniform(it.head), steps = tiles * group;
        int t = 0, h = head * group;
#pragma unroll 1
        for (int j = 0; j < steps; ++j) {
          float lse[4], delta[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int q = t * kTile + lane + 32 * e;
            lse[e] = q < it.rows ? __ldg(a.lse + h * a.q.rows + it.q_row + q) * kLog2e : -INFINITY;
            delta[e] = q < it.rows ? a.delta[h * a.delta_rows + it.q_row + q] : 0.f;
          }
          if (!first && !(ok = bar_wait(b.stat_free + 8 * at.stage, at.parity ^ 1, a.error))) break;
          float* to = reinterpret_cast<float*>(sm + L::kStats + at.stage * L::kStatBytes);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            to[lane + 32 * e] = lse[e] == -INFINITY ? -INFINITY : -lse[e];    // no weight for a row that sees nothing
            to[kTile + lane + 32 * e] = -delta[e];
          }
          bar_arrive_warp(b.stat_full + 8 * at.stage, leader);
          at.next();
          first = first && at.stage;
          if (++t == tiles) {
            t = 0;
            ++h;
          }
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
    Place<L::kStages> at;
    Place<L::kStatStages> st;
    uint32_t n = 0, items = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const AttnTile it = a.k_tile[i];
      if (i + 1 < i1) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.k_tile + i + 1));
      const int tiles = uniform(it.n), steps = tiles * group, queries = uniform(it.rows), first_seen = uniform(it.seen);
      bool ok = true;
      int t = 0;
#pragma unroll 1
      for (int j = 0; j < steps; ++j, ++n) {
        const float* stat = reinterpret_cast<const float*>(sm + L::kStats + st.stage * L::kStatBytes) + c0;
        // queries [from, to) of this half see the key
        const int q0 = t * kTile, rows = queries - q0, from = r + 1 - first_seen - q0 - c0, to = rows - c0;
        const bool tail = rows < kTile, masked = first_seen + q0 < kTile || tail;
        const uint32_t q_stage = at.stage;
        at.next();
        t = t + 1 < tiles ? t + 1 : 0;
        if (!(ok = bar_wait(b.stat_full + 8 * st.stage, st.parity, a.error) && bar_wait(b.s_full, n & 1, a.error))) break;
        fence_after();
        if (masked) keep(S, 64, from, to, -INFINITY);
        float p[64];
        get(S, p);
        weights(p, c2, stat, true);
        put<BF16>(S, p);
        if (tail) {
          if (!(ok = bar_wait(b.full + 8 * at.stage, at.parity, a.error))) break;
          clear_rows<DP>(sm + L::kRing + at.stage * L::kTileBytes, rows);
          clear_rows<DP>(sm + L::kRing + q_stage * L::kTileBytes, rows);     // there since S is
        }
        wait_st();
        fence_before();
        bar_arrive_warp(b.p_ready, leader);
        if (!(ok = bar_wait(b.dp_full, n & 1, a.error))) break;
        fence_after();
        if (tail) keep(Dp, 64, 0, to, 0.f);                   // of rows that may be anything
        float d[64];
        get(Dp, d);
        weight_gradients(d, p, stat + kTile, true);
        put<BF16>(Dp, d);
        wait_st();
        fence_before();
        bar_arrive_warp(b.ds_ready, leader);
        bar_arrive_warp(b.stat_free + 8 * st.stage, leader);
        at.next();
        st.next();
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
  constexpr uint32_t kS = 0, kDp = 128, kDq = 256, kQ = 384, kDo = 448;
  extern __shared__ __align__(1024) uint8_t sm[];
  const uint32_t base = smem_addr(sm);
  const Bars<DP> b(base + L::kBars);
  int* const shared_int = reinterpret_cast<int*>(sm + L::kInts);
  const int warp = uniform(threadIdx.x / 32);
  if (!swizzle_aligned(base, a.error)) return;
  if (threadIdx.x == 0) b.init(8);
  if (warp == 9) tmem_alloc<512>(smem_addr(shared_int));
  const int group = a.heads / a.kv_heads;
  const int i0 = uniform(a.q_first[blockIdx.x]), i1 = uniform(a.q_first[blockIdx.x + 1]);
  asm volatile("prefetch.global.L1 [%0];" ::"l"(a.q_tile + i0));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[0];

  if (warp >= 8) {
    regs_down<kRegsFew>();
    if (warp == 8) {                                        // ---- loads
      Loader<DP> load{base, b, a.error, elect_one()};
      bool ok = true;
#pragma unroll 1
      for (int i = i0; ok && i < i1; ++i) {
        const AttnTile it = a.q_tile[i];
        const int n = uniform(it.n);
        if (!n) continue;
        ok = load.stay(&q_map, &do_map, it.head, (int)it.q_row) && load.pairs(&k_map, &v_map, it.head / group, (int)it.k_row, n);
      }
      load.finish();
    } else if (warp == 9) {                                 // ---- products
      Products<DP, BF16> m(base, tmem, b, a.error, a.dim);
      uint32_t fixed = 0, n = 0;
      // The scores of step j + 1 follow as soon as step j's are in registers,
      // its dO V^T when the product with dS of step j, which replaces dO V^T,
      // is done.
      auto run = [&](int steps) {
        uint32_t k[2], v;                                   // stages of K of this step and the next
#pragma unroll 1
        for (int j = -1; j < steps; ++j) {
          const bool more = j + 1 < steps;
          if (more) {
            if (!(j < 0 ? m.wait(b.fixed_ready, fixed++) : m.wait(b.p_ready, n))) return false;
            if (!m.template across<true>(kS, kQ, b.s_full, k[1])) return false;
          }
          if (j >= 0) {
            if (!m.wait(b.ds_ready, n++)) return false;
            m.gradient(kDq, kDp, k[0], j > 0);
            m.release(k[0]);
          }
          if (more) {
            if (!m.template across<true>(kDp, kDo, b.dp_full, v)) return false;
            m.release(v);
          }
          k[0] = k[1];
        }
        m.done_with(b.out_full);
        return true;
      };
#pragma unroll 1
      for (int i = i0; i < i1; ++i) {
        const int steps = uniform(a.q_tile[i].n);
        if (steps && !run(steps)) break;
      }
      m.done_with(b.done);
      bar_wait(b.done, 0, a.error);
    }
  } else {                                                  // ---- arithmetic: a query per lane, 64 keys
    regs_up<kRegsMany>();
    const bool leader = elect_one();
    const int half = warp / 4, r = threadIdx.x % 128, c0 = 64 * half;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16, S = tmem + lanes + kS + c0, Dp = tmem + lanes + kDp + c0;
    const float c2 = a.scale * kLog2e;
    uint32_t n = 0, items = 0;
    Place<L::kStages> at;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const AttnTile it = a.q_tile[i];
      if (i + 1 < i1) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.q_tile + i + 1));
      const int steps = uniform(it.n), first_seen = uniform(it.seen), keys = uniform(it.keys);
      const int64_t query = it.q_row + r;
      const bool valid = r < it.rows;
      float minus_lse = -INFINITY, minus_delta = 0.f;        // no weight for a row that sees nothing
      if (valid) {
        const float lse = __ldg(a.lse + it.head * a.q.rows + query) * kLog2e;
        minus_lse = lse == -INFINITY ? -INFINITY : -lse;
        minus_delta = -a.delta[it.head * a.delta_rows + query];
      }
      bool ok = true;
      if (steps) {                                            // half of the warps bring Q, half dO
        if (!bar_wait(b.fixed_full, items & 1, a.error)) break;
        tile_to_tmem<DP>(tmem + lanes + (half ? kDo : kQ), sm + half * L::kTileBytes, r);
        fence_before();
        bar_arrive_warp(b.fixed_ready, leader);
        bar_arrive_warp(b.fixed_free, leader);
      }
#pragma unroll 1
      for (int j = 0; j < steps; ++j, ++n) {
        const int seen = first_seen + r - j * kTile - c0;                // keys of this half that the row sees
        const bool masked = (j + 1) * kTile > first_seen;
        if (!(ok = bar_wait(b.s_full, n & 1, a.error))) break;
        fence_after();
        if (masked) keep(S, 64, 0, seen, -INFINITY);
        float p[64];
        get(S, p);
        fence_before();
        bar_arrive_warp(b.p_ready, leader);
        weights(p, c2, &minus_lse, false);
        if (!(ok = bar_wait(b.dp_full, n & 1, a.error))) break;
        fence_after();
        if (masked) keep(Dp, 64, 0, seen, 0.f);               // of keys that may be anything
        float d[64];
        get(Dp, d);
        weight_gradients(d, p, &minus_delta, false);
        put<BF16>(Dp, d);
        if ((j + 1) * kTile > keys) clear_rows<DP>(sm + L::kRing + at.stage * L::kTileBytes, keys - j * kTile);
        wait_st();
        fence_before();
        bar_arrive_warp(b.ds_ready, leader);
        at.next();
        at.next();
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

// delta of every row and head, eight entries per lane; LANES lanes a head.  It
// is of the rounded output, the one that the forward pass leaves: an unrounded
// copy would be twice its bytes, and rowsum(P dP), which equals it, a third walk.
// Its error is shared by a row's dS: in bf16 dq is off by 3.2e-3 at 8 keys and
// 2.5e-3 at 1024 where rounding dq alone takes 1.7e-3.
// Bound by memory: 8192 rows of 32 heads of 128 take 24 us (5.6 TB/s).
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
// once delta is there.)  Tiles that meet nothing are written as zeros at once,
// so a walk starts early only behind the kernel that it expects: the key walk
// behind delta, which started in the plain way, when all earlier work of the
// stream was done, and the query walk behind the key walk.  Without queries
// there is no delta, and what comes before may still read the memory that dk
// and dv now are; without keys delta itself comes before the query walk, which
// reads it.
template <class K>
cudaError_t walk(K kernel, int blocks, int bytes, bool early, std::atomic<uint64_t>& allowed, const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  cudaError_t e = allow_smem(kernel, bytes, allowed);
  if (e != cudaSuccess) return e;
  e = early ? launch_early(kernel, blocks, kThreads, bytes, st, a, m.q, m.k, m.v, m.d_o)
            : launch_plain(kernel, blocks, kThreads, bytes, st, a, m.q, m.k, m.v, m.d_o);
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
  if (a.n_k_blocks && (e = walk(k_attn_dkv<DP, BF16>, a.n_k_blocks, L::kBytes, a.delta_rows > 0, dkv_allowed, a, m, st)) != cudaSuccess) return e;
  if (a.n_q_blocks && (e = walk(k_attn_dq<DP, BF16>, a.n_q_blocks, L::kBytes, a.n_k_blocks > 0, dq_allowed, a, m, st)) != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_attn_backward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  if (a.dim <= 64) return a.bf16 ? launch<64, true>(a, m, st) : launch<64, false>(a, m, st);
  return a.bf16 ? launch<128, true>(a, m, st) : launch<128, false>(a, m, st);
}

}  // namespace syncgb

// Forward attention over packed sequences (include/sync.h, sync_attn_forward).
//
// One block per SM takes work items in turn: two query tiles of 128 rows
// against a range of 128-key tiles, S = Q K^T and O += P V on the tensor
// cores with accumulators in tensor memory.  Warps by role: four for each
// query tile (a thread has a row: running maximum and sum of the softmax
// with no exchange between lanes), one loads tiles, one issues products.
// The two query tiles take turns on the tensor cores: while one's softmax
// runs, the other's products do.  P replaces S in tensor memory as the first
// operand of the second product and never passes through shared memory.
//
// Rows of a tile are consecutive queries of one head, or, where a sequence
// has few queries, the queries of all heads of a group (row = query * group +
// head): their keys are then read once for the group.  A key range that would
// leave SMs idle is split into pieces whose results are merged by whichever
// block finishes last, in the order of the pieces.
#include <algorithm>

#include "attn.h"
#include "umma.cuh"

namespace syncgb {
namespace {

using namespace umma;

constexpr int kThreads = 384;          // two softmax groups of 4 warps; one warp loads, one multiplies, two are idle
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
  static constexpr int kInts = kBars + 104 + 16 * kStages;  // after the barriers: dead, tensor memory, last[2]
  static constexpr int kBytes = kInts + 16 + 1024;          // alignment
};

// What an item asks of query tile t: key tiles, and its rows.
struct Part {
  int n;          // key tiles
  int first;      // first query
  int rows;       // queries
};
__device__ __forceinline__ Part part_of(const AttnItem& it, const AttnSeq& s, int per, int t) {
  Part p;
  p.first = it.q0 + t * per;
  p.rows = max(0, min(per, s.lq - p.first));
  const int seen = max(0, p.first + p.rows + s.lk - s.lq);          // keys that the last row sees
  p.n = p.rows ? max(0, min(it.kt1, (seen + kTile - 1) / kTile) - it.kt0) : 0;
  return p;
}

template <bool BF16>
__device__ __forceinline__ void store8(void* p, const float* x) {
  uint4 v;
  v.x = pack2<BF16>(x[0], x[1]);
  v.y = pack2<BF16>(x[2], x[3]);
  v.z = pack2<BF16>(x[4], x[5]);
  v.w = pack2<BF16>(x[6], x[7]);
  *static_cast<uint4*>(p) = v;
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) k_attn_fwd(const __grid_constant__ AttnArgs a,
                                                          const __grid_constant__ CUtensorMap q_map,
                                                          const __grid_constant__ CUtensorMap qg_map,
                                                          const __grid_constant__ CUtensorMap k_map,
                                                          const __grid_constant__ CUtensorMap v_map) {
  using L = Layout<DP>;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t base = smem_addr(sm), bars = base + L::kBars;
  const uint32_t q_full = bars, q_free = bars + 16, s_full = bars + 32, p_full = bars + 48, o_full = bars + 64,
                 merge = bars + 80, done = bars + 96, full = bars + 104, free_ = full + 8 * L::kStages;
  int* const shared_int = reinterpret_cast<int*>(sm + L::kInts);
  const Waits w{shared_int, a.error};
  int* const last_one = shared_int + 2;
  const int warp = threadIdx.x / 32;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      bar_init(q_full + 8 * t, 1);
      bar_init(q_free + 8 * t, 1);
      bar_init(s_full + 8 * t, 1);
      bar_init(p_full + 8 * t, 4);
      bar_init(o_full + 8 * t, 1);
      bar_init(merge + 8 * t, 128);
    }
    bar_init(done, 1);
    for (int i = 0; i < L::kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(free_ + 8 * i, 1);
    }
    bar_init_visible();
    shared_int[0] = 0;
  }
  if (warp == 9) tmem_alloc<kCols>(smem_addr(shared_int + 1));
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)shared_int[1];

  const int group = a.heads / a.kv_heads, packed_rows = kTile / group;
  const int i0 = a.block_first[blockIdx.x], i1 = a.block_first[blockIdx.x + 1];

  if (warp >= 8) {
    regs_down<kRegsFew>();
    if (warp == 8 && elect_one()) {                         // ---- loads
      uint32_t pos = 0, qn[2] = {0, 0};
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int head, int row) {
        const uint32_t st = pos % L::kStages, bar = full + 8 * st;
        if (pos >= L::kStages && !bar_wait(free_ + 8 * st, (pos / L::kStages - 1) & 1, w)) return false;
        bar_expect(bar, L::kTileBytes);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
          tma_load(base + L::kRing + st * L::kTileBytes + c * kBlockBytes, map, bar, 64 * c, head, row);
        ++pos;
        return true;
      };
      for (int i = i0; ok && i < i1; ++i) {
        const AttnItem it = a.item[i];
        const AttnSeq s = a.seq[it.seq];
        const int per = it.packed ? packed_rows : kTile;
        const int kh = it.head / group;
        const Part p[2] = {part_of(it, s, per, 0), part_of(it, s, per, 1)};
        const int n = max(p[0].n, p[1].n);
        for (int t = 0; ok && t < 2; ++t) {
          if (!p[t].n) continue;
          if (qn[t] && !bar_wait(q_free + 8 * t, (qn[t] - 1) & 1, w)) { ok = false; break; }
          bar_expect(q_full + 8 * t, DP / 64 * (it.packed ? packed_rows * group : kTile) * 128);
#pragma unroll
          for (int c = 0; c < DP / 64; ++c)
            tma_load(base + t * L::kTileBytes + c * kBlockBytes, it.packed ? &qg_map : &q_map, q_full + 8 * t, 64 * c,
                     it.head, (int)s.q0 + p[t].first);
          ++qn[t];
        }
        for (int j = 0; ok && j < n; ++j) {
          const int row = (int)s.k0 + (it.kt0 + j) * kTile;
          ok = load(&k_map, kh, row) && load(&v_map, kh, row);
        }
      }
      // nothing is in flight when the block ends
      for (uint32_t i = pos > L::kStages ? pos - L::kStages : 0; i < pos; ++i)
        bar_wait(full + 8 * (i % L::kStages), i / L::kStages & 1, w);
      for (int t = 0; t < 2; ++t)
        if (qn[t]) bar_wait(q_full + 8 * t, (qn[t] - 1) & 1, w);
    } else if (warp == 9 && elect_one()) {                  // ---- products
      const int ksteps = (a.dim + 15) / 16, n_out = ksteps * 16;
      const uint32_t i_s = instr(BF16, kTile, false), i_o = instr(BF16, n_out, true);
      uint32_t pos = 0, qn[2] = {0, 0}, pn[2] = {0, 0};
      auto tile = [&](uint32_t at) { return tile_desc(base + L::kRing + at % L::kStages * L::kTileBytes); };
      auto arrived = [&](uint32_t at) { return bar_wait(full + 8 * (at % L::kStages), at / L::kStages & 1, w); };
      auto scores = [&](int t, uint32_t at) {
        const uint64_t q = tile_desc(base + t * L::kTileBytes), k = tile(at);
        for (int e = 0; e < ksteps; ++e) mma(tmem + s_col(t), q + step_along(e), k + step_along(e), i_s, e > 0);
        commit(s_full + 8 * t);
      };
      auto run = [&](const Part* p) {
        const int n = max(p[0].n, p[1].n);
        if (!n) return true;
        if (!arrived(pos)) return false;
        for (int t = 0; t < 2; ++t) {
          if (!p[t].n) continue;
          if (!bar_wait(q_full + 8 * t, qn[t]++ & 1, w)) return false;
          fence_after();
          scores(t, pos);
          if (p[t].n == 1) commit(q_free + 8 * t);
        }
        commit(free_ + 8 * (pos % L::kStages));
        for (int j = 0; j < n; ++j, pos += 2) {
          if (!arrived(pos + 1) || (j + 1 < n && !arrived(pos + 2))) return false;
          for (int t = 0; t < 2; ++t) {
            if (j < p[t].n) {
              if (!bar_wait(p_full + 8 * t, pn[t]++ & 1, w)) return false;
              fence_after();
              const uint64_t v = tile(pos + 1);
#pragma unroll
              for (int e = 0; e < kTile / 16; ++e)
                mma_tmem(tmem + o_col(t), tmem + s_col(t) + 8 * e, v + step_rows(e), i_o, j > 0 || e > 0);
              if (j + 1 == p[t].n) commit(o_full + 8 * t);
            }
            if (j + 1 < p[t].n) {
              scores(t, pos + 2);
              if (j + 2 == p[t].n) commit(q_free + 8 * t);
            }
          }
          commit(free_ + 8 * ((pos + 1) % L::kStages));
          if (j + 1 < n) commit(free_ + 8 * ((pos + 2) % L::kStages));
        }
        return true;
      };
      for (int i = i0; i < i1; ++i) {
        const AttnItem it = a.item[i];
        const AttnSeq s = a.seq[it.seq];
        const int per = it.packed ? packed_rows : kTile;
        const Part p[2] = {part_of(it, s, per, 0), part_of(it, s, per, 1)};
        if (!run(p)) break;
      }
      commit(done);
      bar_wait(done, 0, w);
    }
  } else {                                                  // ---- softmax of query tile t
    regs_up<kRegsMany>();
    const int t = warp / 4, r = threadIdx.x % 128;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16, S = tmem + s_col(t) + lanes, O = tmem + o_col(t) + lanes;
    const float c2 = a.scale * 1.4426950408889634f;          // weights are powers of two
    const float slack = 8.f / c2;                            // see below
    uint32_t pos = 0, sn = 0, on = 0, mn = 0;
    for (int i = i0; i < i1; ++i) {
      const AttnItem it = a.item[i];
      const AttnSeq s = a.seq[it.seq];
      const int per = it.packed ? packed_rows : kTile;
      const Part p[2] = {part_of(it, s, per, 0), part_of(it, s, per, 1)};
      const int n = p[t].n, rq = it.packed ? r / group : r;
      const int head = it.packed ? it.head + r % group : it.head;
      const int query = p[t].first + rq, offset = s.lk - s.lq;
      const bool valid = rq < p[t].rows;
      const int last_key = min(query, s.lq - 1) + offset;    // the last one that this row sees
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (int j = 0; j < n; ++j) {
        const int k0 = (it.kt0 + j) * kTile;
        if (!(ok = bar_wait_warp(s_full + 8 * t, sn++ & 1, w))) break;
        fence_after();
        float x[kTile];
#pragma unroll
        for (int c = 0; c < kTile; c += 32) tmem_ld32(S + c, x + c);
        wait_ld();
        if (k0 + kTile - 1 > p[t].first + offset) {           // some row does not see the whole tile
          const int seen = last_key - k0 + 1;
#pragma unroll
          for (int c = 0; c < kTile; ++c) x[c] = c < seen ? x[c] : -INFINITY;
        }
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
        const bool rises = j > 0 && top > m + slack;
        if (j == 0) m = top;
        if (__any_sync(~0u, rises)) {
          const float by = rises ? exp2_fast((m - top) * c2) : 1.f;
          m = rises ? top : m;
          l *= by;
#pragma unroll 1
          for (int c = 0; c < DP; c += 16) {
            float o[16];
            tmem_ld16(O + c, o);
            wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= by;
            tmem_st16(O + c, reinterpret_cast<uint32_t*>(o));
          }
        }
        const float shift = m == -INFINITY ? 0.f : m * c2;
        float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kTile; c += 32) {
          uint32_t y[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float u = exp2_fast(fmaf(x[c + e], c2, -shift)), v = exp2_fast(fmaf(x[c + e + 1], c2, -shift));
            l4[e / 2 % 2] += u;
            l4[2 + e / 2 % 2] += v;
            y[e / 2] = pack2<BF16>(u, v);
          }
          tmem_st16(S + c / 2, y);
        }
        l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
        if (k0 + kTile > s.lk) {
          // The tile ends past the sequence: its values there belong to others
          // and may be anything, so they are cleared (both groups write the
          // same zeros).
          const uint32_t at = pos + 2 * j + 1, st = at % L::kStages;
          if (!(ok = bar_wait_warp(full + 8 * st, at / L::kStages & 1, w))) break;
          uint8_t* v = sm + L::kRing + st * L::kTileBytes;
          for (int b = (s.lk - k0) * 8 + r; b < kTile * 8; b += 128)
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) *reinterpret_cast<uint4*>(v + c * kBlockBytes + b * 16) = make_uint4(0, 0, 0, 0);
          fence_async();
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (threadIdx.x % 32 == 0) bar_arrive(p_full + 8 * t);
      }
      pos += 2 * max(p[0].n, p[1].n);
      if (!ok) break;
      if (n) {
        if (!bar_wait_warp(o_full + 8 * t, on++ & 1, w)) break;
        fence_after();
      }
      const float by = l == 0.f ? 0.f : 1.f / l;
      const float lse2 = l == 0.f ? -INFINITY : fmaf(m, c2, log2f(l));
      if (it.group < 0) {
        uint8_t* out = static_cast<uint8_t*>(a.o.data) + 2 * ((s.q0 + query) * a.o.row + head * a.o.head);
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          float o[32];
          if (n) {
            tmem_ld32(O + c, o);
            wait_ld();
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = n && l != 0.f ? o[e] * by : 0.f;
          if (valid)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              if (c + e < a.dim) store8<BF16>(out + 2 * (c + e), o + e);
        }
        if (valid && a.lse) a.lse[head * a.q.rows + s.q0 + query] = lse2 * 0.6931471805599453f;
        continue;
      }
      // A piece of a split key range: its rows, scaled by its own sum, and
      // their logarithms, for the piece that finishes last.
      const AttnSplit g = a.split[it.group];
      float* part = a.part_o + ((int64_t)(g.slot + it.piece) * 2 + t) * kTile * DP;
      float* part_lse = a.part_lse + ((int64_t)(g.slot + it.piece) * 2 + t) * kTile;
      if (p[t].rows == 0) continue;                           // no piece of this tile has rows
#pragma unroll 1
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (n) {
          tmem_ld32(O + c, o);
          wait_ld();
        }
        if (valid)
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            float4 f = make_float4(o[e] * by, o[e + 1] * by, o[e + 2] * by, o[e + 3] * by);
            if (!n || l == 0.f) f = make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<float4*>(part + r * DP + c + e) = f;
          }
      }
      if (valid) part_lse[r] = lse2;
      __threadfence();
      bar_arrive(merge + 8 * t);
      if (!bar_wait_warp(merge + 8 * t, mn++ & 1, w)) break;
      if (r == 0) {
        const int before = atomicAdd(a.split_count + 2 * it.group + t, 1);
        last_one[t] = before == g.pieces - 1;
        if (before == g.pieces - 1) a.split_count[2 * it.group + t] = 0;
      }
      bar_arrive(merge + 8 * t);
      if (!bar_wait_warp(merge + 8 * t, mn++ & 1, w)) break;
      if (!last_one[t]) continue;
      __threadfence();
      const int lane = threadIdx.x % 32;
      const float* lse0 = a.part_lse + ((int64_t)g.slot * 2 + t) * kTile;
      const float* o0 = a.part_o + ((int64_t)g.slot * 2 + t) * kTile * DP;
      for (int row = warp % 4; row < p[t].rows * (it.packed ? group : 1); row += 4) {
        float top = -INFINITY;
        for (int k = lane; k < g.pieces; k += 32) top = fmaxf(top, __ldcg(lse0 + (int64_t)k * 2 * kTile + row));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        const float from = top == -INFINITY ? 0.f : top;
        float acc[DP / 32], sum = 0.f;
#pragma unroll
        for (int e = 0; e < DP / 32; ++e) acc[e] = 0.f;
#pragma unroll 4
        for (int k = 0; k < g.pieces; ++k) {
          const float f = exp2_fast(__ldcg(lse0 + (int64_t)k * 2 * kTile + row) - from);
          sum += f;
#pragma unroll
          for (int e = 0; e < DP / 32; ++e) acc[e] += f * __ldcg(o0 + ((int64_t)k * 2 * kTile + row) * DP + lane * (DP / 32) + e);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int rq1 = it.packed ? row / group : row, h1 = it.packed ? it.head + row % group : it.head;
        const int64_t at = s.q0 + p[t].first + rq1;
        if (lane * (DP / 32) < a.dim) {
          uint8_t* out = static_cast<uint8_t*>(a.o.data) + 2 * (at * a.o.row + h1 * a.o.head + lane * (DP / 32));
#pragma unroll
          for (int e = 0; e < DP / 32; e += 2) *reinterpret_cast<uint32_t*>(out + 2 * e) = pack2<BF16>(acc[e] * inv, acc[e + 1] * inv);
        }
        if (a.lse && lane == 0) a.lse[h1 * a.q.rows + at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 9) tmem_free<kCols>(tmem);
}

template <int DP, bool BF16>
cudaError_t launch(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  using L = Layout<DP>;
  // set on every call: a device keeps its own value, and the call costs a microsecond at most
  cudaError_t e = cudaFuncSetAttribute(k_attn_fwd<DP, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (e != cudaSuccess) return e;
  k_attn_fwd<DP, BF16><<<a.n_blocks, kThreads, L::kBytes, st>>>(a, m.q, m.q_group, m.k, m.v);
  e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace

cudaError_t launch_attn_forward(const AttnArgs& a, const AttnMaps& m, cudaStream_t st) {
  if (a.dim <= 64) return a.bf16 ? launch<64, true>(a, m, st) : launch<64, false>(a, m, st);
  return a.bf16 ? launch<128, true>(a, m, st) : launch<128, false>(a, m, st);
}

}  // namespace syncgb

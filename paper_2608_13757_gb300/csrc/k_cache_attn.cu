// Attention of a few new tokens per sequence over the paged cache
// (include/sync.h, sync_cache_attn).
//
// The work is one pass over the cached keys and values, bound by memory.  The
// rows that share a key head (heads of the group times new tokens, in passes of
// 8 NT) are the columns of the products: S^T = K Q^T and O^T += V^T P^T in
// instructions of 16 x 8 x 16, with 16 keys (then 16 entries) as rows, so that a
// group of 8 heads wastes nothing where a tile with queries as rows would waste
// half and the 128-row tiles of tcgen05 fifteen sixteenths.  A warp holds 16 keys
// at a time: it copies them to its part of shared memory some tiles ahead, keeps
// the running maximum and sum of its keys, and turns P^T around in registers
// (movmatrix).  The four warps of a block take 16 keys each of a tile of 64 and
// join their results when a piece ends.
//
// Lengths are on the device, so the blocks divide the work themselves: they are as
// many as fit at once, each takes an equal run of tiles of the list sequence >
// key head > pass > tile (every pass counts kUnitCost tiles more, for its start
// and end).  A pass that is cut leaves its pieces' rows in 32 bits, which a second
// kernel joins in order, so the result does not depend on who ran first.
//
// 4 bits.  A stored code n = value / scale + 8 is a float16 as it is: bits 0-3 of
// a half word are n 2^-24 and bits 4-7 are 16 n 2^-24, subnormal numbers that the
// products take exactly.  So a word of 8 codes becomes four operand registers by
// four masks and a shift, the factor 16 is in the query (or comes out of the sum at
// the end), and the 8 is taken off by the sum's start (scores) or by a product
// with -8 (outputs).  Scales of keys multiply the 32-bit sums of their group;
// those of values multiply the weights, scaled to float16's range by a power of
// two that a warp raises when a larger scale comes.
#include <algorithm>
#include <atomic>

#include "cache.h"
#include "division.h"
#include "launch.cuh"
#include "paged.cuh"
#include "rotate.cuh"
#include "umma.cuh"

namespace syncgb {
namespace {

using division::Header;
using division::kTile;
using division::Lister;
using division::Piece;
using division::Shape;
using umma::exp2_fast;
using umma::pack2;
using umma::smem_addr;
using umma::unpack2;

constexpr int kWarps = 4, kThreads = 32 * kWarps, kKeys = 16;
static_assert(kTile == kWarps * kKeys, "a warp has 16 keys of a tile");
constexpr int kPieces = 16;                // of a block's list that are laid out at a time

// Blocks per SM
constexpr int per_sm(int bits, int nt) { return bits == 4 && nt == 1 ? 4 : 2; }

template <int DP, int ROWS>
struct Parts {                             // the workspace
  static constexpr int kRow = DP + 4;      // a row's entries, then its maximum and sum
  static __host__ __device__ size_t header(int blocks) { return ((size_t)blocks * sizeof(Header) + 255) / 256 * 256; }
  static __host__ __device__ size_t bytes(int blocks) { return header(blocks) + (size_t)2 * blocks * ROWS * kRow * sizeof(float); }
};

// ---- instructions ----
template <bool BF16>
__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, const float* c) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t* r) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// 8 x 8 16-bit entries turned around
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// 16 bytes to shared memory without waiting; zeros where `on` is false
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int N>
__device__ __forceinline__ void read_words(uint32_t addr, uint32_t* x) {
  if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
  else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(addr) : "memory");
  else
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x[i]) : "r"(addr + 4 * i) : "memory");
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ uint32_t as_word(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }

// ---- the two formats ----
// Each holds a warp's queries and outputs, copies a tile of 16 keys to shared
// memory, and has the scores of a tile and the products with its values.

template <int DP_, int NT, bool BF16>
struct Wide {                              // 16 bits
  static constexpr int DP = DP_, kStages = 3, kSide = kKeys * DP * 2, kStage = 2 * kSide;
  uint32_t q[DP / 16][NT][2];
  float o[DP / 16][NT][4], f;

  __device__ __forceinline__ void fetch(const CacheArgs& a, uint32_t stage, int64_t row, int keys) const {
    const int lane = threadIdx.x % 32, chunks = a.dim / 8;
#pragma unroll
    for (int e = 0; e < kKeys * DP / 8 / 32; ++e) {
      const int i = lane + 32 * e, key = i / (DP / 8), j = i % (DP / 8);
      const bool on = key < keys && j < chunks;
      const int64_t from = ((row + key) * a.dim + 8 * j) * 2;
      const uint32_t to = stage + key * DP * 2 + ((j ^ key % 8) * 16);
      copy16(to, on ? a.k + from : a.k, on);
      copy16(to + kSide, on ? a.v + from : a.v, on);
    }
  }
  // the query row of column lane / 4; null: none
  __device__ __forceinline__ void queries(const CacheArgs& a, int nt, const uint8_t* row) {
    const int c = threadIdx.x % 4;
    f = a.scale * 1.4426950408889634f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = 16 * k + 8 * e + 2 * c;
        q[k][nt][e] = row && d < a.dim ? __ldg(reinterpret_cast<const uint32_t*>(row + 2 * d)) : 0;
      }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
  }
  __device__ __forceinline__ float factor(int, int) const { return f; }
  __device__ __forceinline__ void scores(uint32_t stage, float (*s)[4]) const {
    const int lane = threadIdx.x % 32, key = lane % 16;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      uint32_t x[4];
      ldmatrix4<false>(stage + key * DP * 2 + (((2 * k + lane / 16) ^ key % 8) * 16), x);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma<BF16>(s[nt], x, q[k][nt][0], q[k][nt][1], s[nt]);
    }
  }
  __device__ __forceinline__ void outputs(uint32_t stage, int, const float (*p)[4]) {
    const int lane = threadIdx.x % 32, key = lane % 8 + lane / 16 * 8;
    uint32_t b[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      b[nt][0] = transposed(pack2<BF16>(p[nt][0], p[nt][1]));
      b[nt][1] = transposed(pack2<BF16>(p[nt][2], p[nt][3]));
    }
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      uint32_t x[4];
      ldmatrix4<true>(stage + kSide + key * DP * 2 + (((2 * i + lane / 8 % 2) ^ key % 8) * 16), x);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma<BF16>(o[i][nt], x, b[nt][0], b[nt][1], o[i][nt]);
    }
  }
  __device__ __forceinline__ void rescale(int nt, int j, float by) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      o[i][nt][j] *= by;
      o[i][nt][j + 2] *= by;
    }
  }
  // f(entry, column 2 c + j, value) for all of this lane's outputs
  template <class F>
  __device__ __forceinline__ void each(int nt, F&& put) const {
    const int r = threadIdx.x % 32 / 4;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) put(16 * i + r + e / 2 * 8, e % 2, o[i][nt][e]);
  }
};

template <int G, int NT, bool BF16>
struct Narrow {                            // 4 bits, G groups of 32 entries
  static constexpr int DP = 32 * G, kStages = 4, kSide = kKeys * 16 * G, kScales = kKeys * 2 * G, kStage = 2 * (kSide + kScales);
  uint32_t q[2 * G][NT][2];
  float start[G][NT][2];                   // -8 sum q of a group
  float o[2 * G][NT][4], off[NT][4];       // off: row w has -8 sum p s of group w
  float f[NT][2];
  uint32_t by;                             // 1 / bound twice, in float16
  float bound;                             // a power of two that no scale so far reaches

  __device__ __forceinline__ void fetch(const CacheArgs& a, uint32_t stage, int64_t row, int keys) const {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int e = 0; e < (kKeys * G + 31) / 32; ++e) {
      const int i = lane + 32 * e, key = i / G, j = i % G;
      if (i >= kKeys * G) break;
      const bool on = key < keys;
      const int64_t from = (row + key) * (16 * G) + 16 * j;
      copy16(stage + 16 * i, on ? a.k + from : a.k, on);
      // rows of values: even keys first, so that the four keys of a product's slots lie side by side
      copy16(stage + kSide + (key / 2 + key % 2 * 8) * 16 * G + 16 * j, on ? a.v + from : a.v, on);
    }
    if (lane < 4 * G) {                    // 2 G pieces of 16 bytes for keys, then for values
      const bool is_v = lane >= 2 * G;
      const int i = is_v ? lane - 2 * G : lane;
      const uint8_t* from = (is_v ? a.v_scale : a.k_scale) + row * (2 * G) + 16 * i;
      copy16(stage + 2 * kSide + (is_v ? kScales : 0) + 16 * i, from, true);
    }
  }
  __device__ __forceinline__ void queries(const CacheArgs& a, int nt, const uint8_t* row) {
    const int lane = threadIdx.x % 32, c = lane % 4;
    float x[G][8];
    float top = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row) v = __ldg(reinterpret_cast<const uint4*>(row + 2 * (32 * w + 8 * c)));
      const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 y = unpack2<BF16>(words[e]);
        x[w][2 * e] = y.x;
        x[w][2 * e + 1] = y.y;
        top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
      }
    }
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
    // the head's largest entry into 2^11 .. 2^12
    const int k = min(100, 11 + 127 - (int)(__float_as_uint(top) >> 23));
    const float up = __uint_as_float((uint32_t)(127 + k) << 23), down = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
    for (int w = 0; w < G; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        q[2 * w + h][nt][0] = pack2<false>(x[w][2 * h] * up, x[w][2 * h + 4] * up);
        q[2 * w + h][nt][1] = pack2<false>(x[w][2 * h + 1] * up * 0.0625f, x[w][2 * h + 5] * up * 0.0625f);
      }
#pragma unroll
    for (int j = 0; j < 2; ++j) f[nt][j] = a.scale * 1.4426950408889634f * 16777216.f * __shfl_sync(~0u, down, (2 * c + j) * 4);
    const uint32_t eight[4] = {0x80088008u, 0x80088008u, 0x80808080u, 0x80808080u};   // -8, and -8 times 16
#pragma unroll
    for (int w = 0; w < G; ++w) {
      float d[4] = {0.f, 0.f, 0.f, 0.f};
      mma<false>(d, eight, q[2 * w][nt][0], q[2 * w][nt][1], d);
      mma<false>(d, eight, q[2 * w + 1][nt][0], q[2 * w + 1][nt][1], d);
      start[w][nt][0] = d[0];
      start[w][nt][1] = d[1];
    }
  }
  __device__ __forceinline__ void clear() {
    by = 0;
    bound = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        off[nt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) o[i][nt][e] = 0.f;
      }
  }
  __device__ __forceinline__ float factor(int nt, int j) const { return f[nt][j]; }
  // the scales of keys r and r + 8, as they lie: G halves each
  static __device__ __forceinline__ void scales(uint32_t at, uint32_t (*x)[(G + 1) / 2]) {
    const int r = threadIdx.x % 32 / 4;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t from = at + (r + 8 * e) * 2 * G;
      if constexpr (G % 2 == 0) {
        read_words<G / 2>(from, x[e]);
      } else {
#pragma unroll
        for (int i = 0; i < (G + 1) / 2; ++i) {
          uint16_t lo, hi = 0;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(lo) : "r"(from + 4 * i) : "memory");
          if (2 * i + 1 < G) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(hi) : "r"(from + 4 * i + 2) : "memory");
          x[e][i] = lo | (uint32_t)hi << 16;
        }
      }
    }
  }
  __device__ __forceinline__ void scores(uint32_t stage, float (*s)[4]) const {
    const int lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
    uint32_t x[2][G], sc[2][(G + 1) / 2];
    read_words<G>(stage + r * 16 * G + 4 * G * c, x[0]);
    read_words<G>(stage + (r + 8) * 16 * G + 4 * G * c, x[1]);
    scales(stage + 2 * kSide, sc);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      const uint32_t lo[4] = {x[0][w] & 0x000f000fu, x[1][w] & 0x000f000fu, x[0][w] & 0x00f000f0u, x[1][w] & 0x00f000f0u};
      const uint32_t y0 = x[0][w] >> 8, y1 = x[1][w] >> 8;
      const uint32_t hi[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
      const float2 k0 = __half22float2(as_half2(sc[0][w / 2])), k1 = __half22float2(as_half2(sc[1][w / 2]));
      const float u0 = w % 2 ? k0.y : k0.x, u1 = w % 2 ? k1.y : k1.x;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float d[4] = {start[w][nt][0], start[w][nt][1], start[w][nt][0], start[w][nt][1]};
        mma<false>(d, lo, q[2 * w][nt][0], q[2 * w][nt][1], d);
        mma<false>(d, hi, q[2 * w + 1][nt][0], q[2 * w + 1][nt][1], d);
        s[nt][0] = fmaf(u0, d[0], s[nt][0]);
        s[nt][1] = fmaf(u0, d[1], s[nt][1]);
        s[nt][2] = fmaf(u1, d[2], s[nt][2]);
        s[nt][3] = fmaf(u1, d[3], s[nt][3]);
      }
    }
  }
  __device__ __forceinline__ void outputs(uint32_t stage, int keys, const float (*p)[4]) {
    const int lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
    uint32_t sc[2][(G + 1) / 2];
    scales(stage + 2 * kSide + kScales, sc);
    if (keys < kKeys) {                    // past the sequence's end a scale may be anything, and a zero weight does not hide a NaN
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < (G + 1) / 2; ++i) sc[e][i] = r + 8 * e < keys ? sc[e][i] : 0;
    }
    __half2 most = __hmax2(as_half2(sc[0][0]), as_half2(sc[1][0]));
    if constexpr (G > 2) most = __hmax2(most, __hmax2(as_half2(sc[0][1]), as_half2(sc[1][1])));
    float top = fmaxf(__low2float(most), __high2float(most));
    if (__any_sync(~0u, top >= bound)) {                     // a larger scale than any so far (or the first tile)
#pragma unroll
      for (int e = 4; e < 32; e *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, e));
      // the power of two above it, from 2^-13 on, so that 1 / bound is a float16
      const float next = fmaxf(bound, __uint_as_float(max(__float_as_uint(top) >> 23, 127u - 14u) + 1 << 23));
      const float ratio = bound / next;
      bound = next;
      by = pack2<false>(1.f / next, 1.f / next);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          off[nt][e] *= ratio;
#pragma unroll
          for (int i = 0; i < 2 * G; ++i) o[i][nt][e] *= ratio;
        }
    }
    __half2 rel[2][(G + 1) / 2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < (G + 1) / 2; ++i) rel[e][i] = __hmul2(as_half2(sc[e][i]), as_half2(by));
    __half2 h[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      h[nt][0] = as_half2(pack2<false>(p[nt][0], p[nt][1]));
      h[nt][1] = as_half2(pack2<false>(p[nt][2], p[nt][3]));
    }
    uint32_t x[4][G];                                        // keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
    for (int e = 0; e < 4; ++e) read_words<G>(stage + kSide + (c + e / 2 * 4 + e % 2 * 8) * 16 * G + 4 * G * (r / 2), x[e]);
    const uint32_t halves = r % 2 ? 0x7632u : 0x5410u;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      uint32_t b[NT][2];
      const __half2 r0 = w % 2 ? __high2half2(rel[0][w / 2]) : __low2half2(rel[0][w / 2]);
      const __half2 r1 = w % 2 ? __high2half2(rel[1][w / 2]) : __low2half2(rel[1][w / 2]);
      const uint32_t mark = r == w ? 0x80088008u : 0u;       // -8 in row w
      const uint32_t eight[4] = {mark, 0u, mark, 0u};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        b[nt][0] = transposed(as_word(__hmul2(h[nt][0], r0)));
        b[nt][1] = transposed(as_word(__hmul2(h[nt][1], r1)));
        mma<false>(off[nt], eight, b[nt][0], b[nt][1], off[nt]);
      }
      const uint32_t y0 = __byte_perm(x[0][w], x[1][w], halves), y1 = __byte_perm(x[2][w], x[3][w], halves);
      const uint32_t lo[4] = {y0 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x000f000fu, y1 & 0x00f000f0u};
      const uint32_t z0 = y0 >> 8, z1 = y1 >> 8;
      const uint32_t hi[4] = {z0 & 0x000f000fu, z0 & 0x00f000f0u, z1 & 0x000f000fu, z1 & 0x00f000f0u};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma<false>(o[2 * w][nt], lo, b[nt][0], b[nt][1], o[2 * w][nt]);
        mma<false>(o[2 * w + 1][nt], hi, b[nt][0], b[nt][1], o[2 * w + 1][nt]);
      }
    }
  }
  __device__ __forceinline__ void rescale(int nt, int j, float by_) {
    off[nt][j] *= by_;
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
      o[i][nt][j] *= by_;
      o[i][nt][j + 2] *= by_;
    }
  }
  template <class F>
  __device__ __forceinline__ void each(int nt, F&& put) const {
    const int lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
    const float unit = bound * 16777216.f;
#pragma unroll
    for (int w = 0; w < G; ++w)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float minus = __shfl_sync(~0u, off[nt][j], 4 * w + c);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          put(32 * w + 4 * r + 2 * h, j, (o[2 * w + h][nt][j] + minus) * unit);
          put(32 * w + 4 * r + 2 * h + 1, j, fmaf(o[2 * w + h][nt][j + 2], 0.0625f, minus) * unit);
        }
      }
  }
};

// ---- division of the work ----
__device__ __forceinline__ Shape shape_of(const CacheArgs& a, int s, int rows) {
  const int64_t begin = a.starts ? __ldg(a.starts + s) : s, end = a.starts ? __ldg(a.starts + s + 1) : s + 1;
  return division::shape(begin, end, a.rows, __ldg(a.lens + s), a.max_pages << a.page_shift, a.heads / a.kv_heads, a.kv_heads, rows);
}

// Where a block's run of the list begins: the sequence, and how far into its
// work.  left: the length of the run.
struct Start {
  int s;
  int64_t into, left;
};

template <int ROWS>
__device__ __forceinline__ Start find_start(const CacheArgs& a, int64_t* shared) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int64_t total = 0;
  for (int s = threadIdx.x; s < a.n_seqs; s += kThreads) total += shape_of(a, s, ROWS).cost;
#pragma unroll
  for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
  if (lane == 0) shared[warp] = total;
  if (threadIdx.x == 0) shared[4] = -1;
  __syncthreads();
  total = shared[0] + shared[1] + shared[2] + shared[3];
  Start r;
  const int takers = division::takers(total, gridDim.x);
  const int64_t x0 = division::bound(total, takers, blockIdx.x);
  r.left = division::bound(total, takers, blockIdx.x + 1) - x0;
  r.s = 0;
  r.into = 0;
  if (r.left == 0) return r;               // (the same for the whole block)
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kThreads) {
    const int s = s0 + threadIdx.x;
    const int64_t cost = s < a.n_seqs ? shape_of(a, s, ROWS).cost : 0;
    int64_t sum = cost;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int64_t up = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += up;
    }
    __syncthreads();
    if (lane == 31) shared[warp] = sum;
    __syncthreads();
    int64_t mine = before + sum - cost;
    for (int w = 0; w < warp; ++w) mine += shared[w];
    before += shared[0] + shared[1] + shared[2] + shared[3];
    if (cost && mine <= x0 && x0 < mine + cost) {
      shared[4] = s;
      shared[5] = x0 - mine;
    }
    __syncthreads();
    if (shared[4] >= 0) break;
  }
  r.s = (int)max(shared[4], (int64_t)0);
  r.into = shared[5];
  __syncthreads();
  return r;
}

template <class K, int NT, bool BF16>
__global__ void __launch_bounds__(kThreads, per_sm(K::kStages == 4 ? 4 : 16, NT)) k_cache_attn(const __grid_constant__ CacheArgs a) {
  constexpr int DP = K::DP, ROWS = 8 * NT, S = K::kStages;
  using P = Parts<DP, ROWS>;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float joined[2][8][DP + 4];
  __shared__ float stat[kWarps][ROWS][2];
  __shared__ Piece list[kPieces];
  __shared__ int64_t scan[6];
  __shared__ int listed;
  __shared__ Lister lister;
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
  const int group = a.heads / a.kv_heads;
  const uint32_t mine = smem_addr(ring) + warp * S * K::kStage;
  Header* const headers = reinterpret_cast<Header*>(a.work);
  float* const parts = reinterpret_cast<float*>(a.work + P::header(gridDim.x));

  if (a.fill) {                            // padding behind the last sequence
    const int64_t end = a.starts ? min(max((int64_t)__ldg(a.starts + a.n_seqs), (int64_t)0), a.rows) : a.rows;
    for (int64_t row = end + blockIdx.x; row < a.rows; row += gridDim.x)
      for (int i = threadIdx.x; i < a.heads * (a.dim / 8); i += kThreads) {
        const int h = i / (a.dim / 8), d = i % (a.dim / 8) * 8;
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.q_out.data) + 2 * (row * a.q_out.row + h * a.q_out.head + d)) = make_uint4(0, 0, 0, 0);
        if (a.lse && d == 0) a.lse[h * a.rows + row] = -INFINITY;
      }
  }

  // the list of pieces is laid out by one thread, kPieces at a time
  const Start at = find_start<ROWS>(a, scan);
  if (threadIdx.x == 0) {
    lister.left = 0;
    lister.header = Header{0, 0, 0, 0, 0, 0};
    if (at.left) lister.start(shape_of(a, at.s, ROWS), at.s, at.into, at.left);
  }
  K k;
  for (;;) {
    if (threadIdx.x == 0) {
      int n = 0;
      while (n < kPieces && lister.next([&](int s) { return shape_of(a, s, ROWS); }, a.n_seqs, a.kv_heads, ROWS, list[n])) ++n;
      listed = n;
    }
    __syncthreads();
    const int pieces = listed;
    if (pieces == 0) break;

    // Tiles ahead: (ap, t) is the next one to copy, its page looked up one tile
    // before.
    int ap = 0, t = list[0].from, page = -1;
    bool bad = false;
    auto settle = [&] {                    // past pieces without tiles
      while (ap < pieces && t >= list[ap].to)
        if (++ap < pieces) t = list[ap].from;
    };
    auto look = [&] {
      if (ap >= pieces) return;
      const int pos = t * kTile + warp * kKeys;
      page = pos < list[ap].len ? __ldg(a.table + list[ap].s * a.table_stride + (pos >> a.page_shift)) : -1;
    };
    int put = 0;
    uint32_t lost = 0;                     // stages whose page the cache does not have
    auto ahead = [&] {
      if (ap < pieces) {
        const int pos = t * kTile + warp * kKeys, keys = list[ap].len - pos;
        if (keys > 0) {
          const bool has = (unsigned)page < (unsigned)a.n_pages;
          lost = has ? lost & ~(1u << put) : lost | 1u << put;
          const int64_t row = (((int64_t)(has ? page : 0) * a.kv_heads + list[ap].head) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
          if (has) k.fetch(a, mine + put * K::kStage, row, min(keys, kKeys));
        }
        ++t;
        settle();
        look();
      }
      end_group();
      put = put + 1 == S ? 0 : put + 1;
    };
    settle();
    look();
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) ahead();
    int get = 0;

#pragma unroll 1
    for (int ip = 0; ip < pieces; ++ip) {
      const Piece x = list[ip];
      float m[NT][2], l[NT][2];
      int limit[NT][2];                    // tokens that a column's row sees
      int least = x.len;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = x.first + 8 * nt + r;
        const bool is = row < x.n * group;
        const int token = row / group, head = x.head * group + row % group;
        k.queries(a, nt, is ? static_cast<const uint8_t*>(a.q.data) + 2 * ((x.row0 + token) * a.q.row + head * a.q.head) : nullptr);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          m[nt][j] = -INFINITY;
          l[nt][j] = 0.f;
          limit[nt][j] = x.len - x.n + min((x.first + 8 * nt + 2 * c + j) / group, x.n - 1) + 1;
          least = min(least, limit[nt][j]);
        }
      }
      k.clear();
      bad = x.bad;
      const bool all = __all_sync(~0u, least == x.len);
#pragma unroll 1
      for (int tile = x.from; tile < x.to; ++tile) {
        __syncwarp();
        ahead();
        wait_groups<S - 1>();
        __syncwarp();
        const uint32_t stage = mine + get * K::kStage;
        const int pos = tile * kTile + warp * kKeys;
        const bool gone = lost >> get & 1;
        get = get + 1 == S ? 0 : get + 1;
        if (pos >= x.len) continue;
        if (gone) {
          bad = true;
          continue;
        }
        float s[NT][4];
        k.scores(stage, s);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][e] *= k.factor(nt, e % 2);
        if (!all || pos + kKeys > x.len) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = pos + r + e / 2 * 8 < limit[nt][e % 2] ? s[nt][e] : -INFINITY;
        }
        // The running maximum follows only rises of more than 2^8 in the weights.
        bool rises = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) rises = rises || fmaxf(s[nt][j], s[nt][j + 2]) > m[nt][j] + 8.f;
        if (__any_sync(~0u, rises)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float top = fmaxf(s[nt][j], s[nt][j + 2]);
#pragma unroll
              for (int o = 4; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
              if (top > m[nt][j] + 8.f) {
                const float by = exp2_fast(m[nt][j] - top);
                m[nt][j] = top;
                l[nt][j] *= by;
                k.rescale(nt, j, by);
              }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float shift = m[nt][e % 2] == -INFINITY ? 0.f : m[nt][e % 2];
            s[nt][e] = exp2_fast(s[nt][e] - shift);
            l[nt][e % 2] += s[nt][e];
          }
        k.outputs(stage, x.len - pos, s);
      }
      // ---- the warps' results joined
      const bool any_bad = __any_sync(~0u, bad);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int o = 4; o < 32; o *= 2) l[nt][j] += __shfl_xor_sync(~0u, l[nt][j], o);
          if (any_bad) l[nt][j] = __int_as_float(0x7fffffff);
          if (r == 0) {
            stat[warp][8 * nt + 2 * c + j][0] = m[nt][j];
            stat[warp][8 * nt + 2 * c + j][1] = l[nt][j];
          }
        }
      __syncthreads();
      const bool whole = x.from == 0 && x.to == x.tiles;
      const int slot = 2 * blockIdx.x + (x.from == 0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {                      // warps 2 and 3, then 0 and 1 on top of them
        float w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int col = 8 * nt + 2 * c + j;
          const float top = fmaxf(fmaxf(stat[0][col][0], stat[1][col][0]), fmaxf(stat[2][col][0], stat[3][col][0]));
          w[j] = m[nt][j] == -INFINITY ? 0.f : exp2_fast(m[nt][j] - top);
        }
        if (warp >= 2) k.each(nt, [&](int d, int j, float v) { joined[warp - 2][2 * c + j][d] = v * w[j]; });
        __syncthreads();
        if (warp < 2) k.each(nt, [&](int d, int j, float v) { joined[warp][2 * c + j][d] += v * w[j]; });
        __syncthreads();
        constexpr int kEach = DP / 16;
        const int col = threadIdx.x / 16, d0 = threadIdx.x % 16 * kEach, row = x.first + 8 * nt + col;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) top = fmaxf(top, stat[i][8 * nt + col][0]);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          const float mi = stat[i][8 * nt + col][0], li = stat[i][8 * nt + col][1];
          sum += mi == -INFINITY ? li : li * exp2_fast(mi - top);      // (li is 0 or NaN then)
        }
        if (!whole) {
          float* to = parts + ((int64_t)slot * ROWS + 8 * nt + col) * P::kRow;
#pragma unroll
          for (int i = 0; i < kEach; ++i) to[d0 + i] = joined[0][col][d0 + i] + joined[1][col][d0 + i];
          if (d0 == 0) {
            to[DP] = top;
            to[DP + 1] = sum;
          }
        } else if (row < x.n * group) {
          const int64_t at_row = x.row0 + row / group;
          const int head = x.head * group + row % group;
          uint8_t* to = static_cast<uint8_t*>(a.q_out.data) + 2 * (at_row * a.q_out.row + head * a.q_out.head);
          const float by = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
          for (int i = 0; i < kEach; i += 2)
            if (d0 + i < a.dim)
              *reinterpret_cast<uint32_t*>(to + 2 * (d0 + i)) =
                  pack2<BF16>((joined[0][col][d0 + i] + joined[1][col][d0 + i]) * by, (joined[0][col][d0 + i + 1] + joined[1][col][d0 + i + 1]) * by);
          if (a.lse && d0 == 0) a.lse[head * a.rows + at_row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        }
        __syncthreads();
      }
    }
    wait_groups<0>();
    __syncthreads();
  }
  if (threadIdx.x == 0) headers[blockIdx.x] = lister.header;
}

// Passes that were cut, from their pieces in order: a block for each block of
// the first kernel that began one, and each of its rows.
template <int DP, int ROWS, bool BF16>
__global__ void __launch_bounds__(kThreads) k_cache_merge(const __grid_constant__ CacheArgs a, int blocks) {
  using P = Parts<DP, ROWS>;
  constexpr int kEach = DP / 32;
  __shared__ float sums[kWarps][DP + 2];
  after_previous();
  const Header* const headers = reinterpret_cast<const Header*>(a.work);
  const Header x = headers[blockIdx.x];
  const int group = a.heads / a.kv_heads, row = x.first + (int)blockIdx.y;
  if (!x.open || row >= x.n * group) return;
  const float* const parts = reinterpret_cast<const float*>(a.work + P::header(blocks)) + blockIdx.y * P::kRow;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int last = blockIdx.x + 1;                                // the block that ends the pass
  for (; last < blocks; last += 32) {
    const uint32_t ends = __ballot_sync(~0u, last + lane < blocks && headers[last + lane].before == 2);
    if (ends) {
      last += __ffs(ends) - 1;
      break;
    }
  }
  last = min(last, blocks - 1);
  auto part = [&](int b) { return parts + (int64_t)(2 * b + (b == (int)blockIdx.x)) * ROWS * P::kRow; };
  float top = -INFINITY;
  for (int b = blockIdx.x + lane; b <= last; b += 32) top = fmaxf(top, part(b)[DP]);
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  float acc[kEach], sum = 0.f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll 4
  for (int b = blockIdx.x + warp; b <= last; b += kWarps) {
    const float* p = part(b);
    const float m = p[DP], f = m == -INFINITY ? 0.f : exp2_fast(m - top), l = p[DP + 1];
    sum += m == -INFINITY ? l : l * f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] = fmaf(f, p[lane * kEach + e], acc[e]);
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) sums[warp][lane * kEach + e] = acc[e];
  if (lane == 0) sums[warp][DP] = sum;
  __syncthreads();
  sum = (sums[0][DP] + sums[1][DP]) + (sums[2][DP] + sums[3][DP]);
  const float by = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t at_row = x.row0 + row / group;
  const int head = x.head * group + row % group, d = 2 * threadIdx.x;
  if (d < a.dim) {
    const float u = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]), v = (sums[0][d + 1] + sums[1][d + 1]) + (sums[2][d + 1] + sums[3][d + 1]);
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.q_out.data) + 2 * (at_row * a.q_out.row + head * a.q_out.head + d)) = pack2<BF16>(u * by, v * by);
  }
  if (a.lse && threadIdx.x == 0) a.lse[head * a.rows + at_row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

template <class K, int NT, bool BF16>
cudaError_t launch(const CacheArgs& a, cudaStream_t st) {
  constexpr int kBytes = kWarps * K::kStages * K::kStage;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = umma::allow_smem(k_cache_attn<K, NT, BF16>, kBytes, allowed);
  if (e != cudaSuccess) return e;
  k_cache_attn<K, NT, BF16><<<a.blocks, kThreads, kBytes, st>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  count_launch();
  e = launch_early(k_cache_merge<K::DP, 8 * NT, BF16>, dim3((unsigned)a.blocks, 8 * NT), kThreads, 0, st, a, a.blocks);
  if (e == cudaSuccess) count_launch();
  return e;
}

template <int NT, bool BF16>
cudaError_t launch_rows(const CacheArgs& a, cudaStream_t st) {
  if (a.bits == 16) return a.dim <= 64 ? launch<Wide<64, NT, BF16>, NT, BF16>(a, st) : launch<Wide<128, NT, BF16>, NT, BF16>(a, st);
  if constexpr (NT <= 2) {
    switch (a.dim / kGroup) {
      case 1: return launch<Narrow<1, NT, BF16>, NT, BF16>(a, st);
      case 2: return launch<Narrow<2, NT, BF16>, NT, BF16>(a, st);
      case 3: return launch<Narrow<3, NT, BF16>, NT, BF16>(a, st);
      default: return launch<Narrow<4, NT, BF16>, NT, BF16>(a, st);
    }
  }
  return cudaErrorInvalidValue;
}

template <bool BF16>
cudaError_t launch_type(const CacheArgs& a, cudaStream_t st) {
  if (a.most_rows == 8) return launch_rows<1, BF16>(a, st);
  if (a.most_rows == 16) return launch_rows<2, BF16>(a, st);
  return launch_rows<4, BF16>(a, st);
}

}  // namespace

int cache_attn_rows(int bits, int group, int max_new) {
  const int64_t rows = (int64_t)group * max_new;
  return rows <= 8 ? 8 : rows <= 16 || bits == 4 ? 16 : 32;
}

int cache_attn_blocks(int bits, int most_rows, int num_sms) { return per_sm(bits, most_rows / 8) * num_sms; }

int64_t cache_attn_workspace(int dim, int most_rows, int blocks) {
  const int dp = dim <= 64 ? 64 : 128;
  const size_t header = Parts<128, 32>::header(blocks);
  return (int64_t)(header + (size_t)2 * blocks * most_rows * (dp + 4) * sizeof(float));
}

cudaError_t launch_cache_attn(const CacheArgs& a, cudaStream_t st) {
  return a.bf16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace syncgb

// Attention of a few new tokens per sequence over the paged cache
// (include/sync.h, sync_cache_attn), or over plain rows of keys and values (plans
// of sync_cross_attn_plan whose sequences have few queries).
//
// The work is one pass over the cached keys and values, bound by memory.  The
// rows that share a key head (heads of the group times new tokens, in passes of
// 8 NT) are the columns of the products: S^T = K Q^T and O^T += V^T P^T in
// instructions of 16 x 8 x 16, with 16 keys (then 16 entries) as rows, so that a
// group of 8 heads wastes nothing where a tile with queries as rows would waste
// half and the 128-row tiles of tcgen05 fifteen sixteenths.  A warp takes 16 keys
// at a time (32 in 4 bits: 524287 keys 134 us, 153 with 16 keys and four blocks an
// SM), works alone, and so waits for no other: it copies tiles to its part of
// shared memory two ahead, keeps the running maximum and sum of its keys, and
// turns P^T around in registers (movmatrix).
//
// Lengths are on the device, so the warps divide the work themselves: the blocks
// are as many as fit at once, each warp takes an equal run of tiles of the list
// sequence > key head > pass > tile (division.h).  A pass that is cut leaves its
// pieces' rows in 32 bits; the block joins those of its warps, a second kernel
// those of the blocks, always in order, so the result does not depend on who ran
// first.  (Joined by the block that ends last instead of by a kernel: one sequence
// of 1802 tokens 14.2 us against 10.3, 131072 tokens in 4 bits 52 against 45.)
//
// Measured, 8 key heads of 128 and 4 queries for each: 16 bits 524287 tokens
// 307 us, 7.0 TB/s; 64 sequences of 1 to 8192 tokens 62.5 us, 5.6 TB/s.  4 bits
// 524287 tokens 126 us, 4.8 TB/s, and 5.6 TB/s for what longer sequences add.  Nothing
// is saturated there (128 sequences of 1 to 16384 tokens: issue slots 53%, DRAM 52%):
// from one instruction of a warp to the next pass 5.4 cycles, 1.6 of them for the
// result before it, 1.5 for the scheduler, a pipe or dispatch, 0.7 for shared or
// global memory, and 2.8 warps a scheduler do not cover that.  Passes of 16 columns
// are further off, with 8 warps an SM and all codes taken apart for every 16 rows: 64
// sequences of 1 to 8192 tokens with up to 4 new ones 51 us, where memory would take
// 9.  One token over one key takes 6 us, over 1024 10 (16 bits) and 13 (4 bits):
// finding the runs 2 us, the first tiles 6, the second kernel 5 after the last block.
//
// 4 bits.  A stored code n = value / scale + 8 is a float16 as it is: bits 0-3 of
// a half word are n 2^-24 and bits 4-7 are 16 n 2^-24, subnormal numbers that the
// products take.  So a word of 8 codes becomes four operand registers by four masks
// and a shift, and the factor 16 is in the query or comes out of the sum at the end.
// The 8 is taken off by the sum's start (scores) or by a product with -8 behind each
// with codes (outputs), so that nothing larger than the result is carried along: -8
// summed for itself and added at the end left rows of 16384 equal weights wrong by
// 1.4%, of 65536 by 2.4%.  Subnormal products are lined up with the others of their 16
// tokens as if they were at 2^-14, and cut there: at about 2^-15 of a code's step of
// the largest weight times scale among them, alike for codes and -8, so that a code
// that stands for 0 leaves nothing.
//
// Scales of keys multiply the 32-bit sums of their group; those of values multiply
// the weights in float16, relative to a power of two for each group that a warp
// raises when a larger scale comes.  (One for the whole head, and weights that were
// not lifted (kLift), took 3 us of 80 less for 128 sequences of 1 to 16384 tokens,
// and lost what many small weights add together: 12 nats below a first token that
// takes the row, 8192 others in a group of a 128th of the head's largest scale left
// 13 to 27% of the result wrong; now it is a rounding of the result.  Products in 32
// bits, rounded once, took 84 us.)
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "cache.h"
#include "division.h"
#include "launch.cuh"
#include "paged.cuh"
#include "rotate.cuh"
#include "umma.cuh"

namespace syncgb {
namespace {

using division::Lister;
using division::Piece;
using division::Shape;
using umma::exp2_fast;
using umma::pack2;
using umma::smem_addr;
using umma::unpack2;

constexpr int kWarps = 4, kThreads = 32 * kWarps, kKeys = 16;
constexpr int kPieces = 8;                 // of a warp's list that are laid out at a time
// The running maximum follows only rises of more than 2^kLag in the weights, whose
// largest then stands for 2^kLift .. 2^(kLift + kLag), the upper end of float16, so
// that smaller ones keep all bits down to 2^-25 of it and are off by 2^-36 of it at
// most below.  Scores past kSure are not lifted: half a unit in their last place is a
// factor that takes the room.
constexpr float kLag = 4.f, kLift = 11.f, kSure = 4194304.f;

// Blocks per SM
constexpr int per_sm(int bits, int nt) { return bits == 4 && nt == 1 ? 3 : 2; }

// What a block leaves for the kernel that joins the pieces: the pass that it has
// begun and does not end, and the block that does.
struct alignas(kWorkAlign) Header {
  int open;                                // 0: none
  int last, row0, n, head, first;          // as in Piece
};
static_assert(alignof(Header) == kWorkAlign && sizeof(Header) % kWorkAlign == 0, "headers lie one after the other from the workspace's start");

template <int DP, int ROWS>
struct Parts {                             // the workspace
  static constexpr int kRow = DP + 4;      // a row's entries, then its maximum and sum
  static constexpr int kFloats = ROWS * kRow;
  static_assert(kRow * sizeof(float) % kWorkAlign == 0, "rows are read and written 16 bytes at a time");
  static __host__ __device__ size_t header(int blocks) { return ((size_t)blocks * sizeof(Header) + 255) / 256 * 256; }
  // two slots per block, then one per warp
  static __device__ int64_t slot(int i) { return (int64_t)i * kFloats; }
  static __device__ int64_t warp_slot(int blocks, int i) { return (int64_t)(2 * blocks + i) * kFloats; }
  static constexpr int kSlots = 2 + kWarps;   // per block
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
// 16 bytes to shared memory without waiting; zeros where `on` is false.  Offsets
// that are known go into the instructions.
template <int TO, int FROM>
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src) {
  asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int N, int AT>
__device__ __forceinline__ void read_words(uint32_t addr, uint32_t* x) {
  if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4 + %5];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr), "n"(AT) : "memory");
  else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2 + %3];" : "=r"(x[0]), "=r"(x[1]) : "r"(addr), "n"(AT) : "memory");
  else {                                   // one by one: three words are aligned to one
    asm volatile("ld.shared.u32 %0, [%1 + %2];" : "=r"(x[0]) : "r"(addr), "n"(AT) : "memory");
    if constexpr (N == 3) {
      read_words<1, AT + 4>(addr, x + 1);
      read_words<1, AT + 8>(addr, x + 2);
    }
  }
}
template <int AT>
__device__ __forceinline__ uint32_t read_half(uint32_t addr) {
  uint16_t x;
  asm volatile("ld.shared.u16 %0, [%1 + %2];" : "=h"(x) : "r"(addr), "n"(AT) : "memory");
  return x;
}
// f with 0, 1, .. as constants
template <int I>
struct Constant {
  static constexpr int value = I;
};
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(Constant<I>());
    unrolled<N, I + 1>(f);
  }
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ uint32_t as_word(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }

// ---- the two formats ----
// Each holds a warp's queries and outputs, copies a tile of 16 keys to shared
// memory, and has the scores of a tile and the products with its values.

template <int DP_, int NT, bool BF16, bool PAGED>
struct Wide {                              // 16 bits; plain rows where not PAGED
  static constexpr int kBits = 16;
  static constexpr bool kPaged = PAGED;
  static constexpr int DP = DP_, MT = 1, kStages = 3, kSide = kKeys * DP * 2, kStage = 2 * kSide;
  uint32_t q[DP / 16][NT][2];
  float o[DP / 16][NT][4], f;

  // What the copies of a tile of 16 keys start from: the keys' and values' first
  // row (in the cache: its row16-th 16 of them), and this lane's part of it.
  using Step = std::conditional_t<PAGED, int, int64_t>;
  Step k, v, k_step, v_step;               // bytes; from one row to the next
  uint32_t to;
  __device__ __forceinline__ void begin(const CacheArgs& a, uint32_t ring) {
    const int lane = threadIdx.x % 32, key = lane / (DP / 8), j = lane % (DP / 8);
    k_step = (Step)(PAGED ? 2 * a.dim : 2 * a.k_rows.row);
    v_step = (Step)(PAGED ? 2 * a.dim : 2 * a.v_rows.row);
    k = key * k_step + 16 * j;
    v = key * v_step + 16 * j;
    to = key * DP * 2 + ((j ^ key) * 16);
    if (a.dim < DP)                        // entries that the heads do not have: zero, and never written again
      for (int i = lane; i < kStages * kStage / 16; i += 32) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring + 16 * i), "r"(0) : "memory");
    __syncwarp();
  }
  template <int T>
  __device__ __forceinline__ void fetch(const CacheArgs& a, uint32_t stage, uint32_t row16, int keys) const {
    const uint64_t at = (uint64_t)row16 * (uint32_t)(32 * a.dim);
    copy(a, stage, a.k + at, a.v + at, keys);
  }
  __device__ __forceinline__ void copy(const CacheArgs& a, uint32_t stage, const uint8_t* rows_k, const uint8_t* rows_v, int keys) const {
    constexpr int kStep = 256 / DP;        // keys that the lanes copy at a time
    const int lane = threadIdx.x % 32, key = lane / (DP / 8), j = lane % (DP / 8);
    if (j >= a.dim / 8) return;
    const uint8_t *from_k = rows_k + k, *from_v = rows_v + v;
#pragma unroll
    for (int e = 0; e < kKeys / kStep; ++e) {
      const uint32_t at = stage + e * kStep * DP * 2 + (to ^ (e * kStep % 8 * 16));
      const uint8_t *at_k = from_k + e * kStep * k_step, *at_v = from_v + e * kStep * v_step;
      if (keys >= kKeys) {
        copy16<0, 0>(at, at_k);
        copy16<kSide, 0>(at, at_v);
      } else {                             // past the sequence's end anything may lie, and a zero weight does not hide a NaN
        const bool on = key + e * kStep < keys;
        copy16(at, on ? at_k : rows_k, on);
        copy16(at + kSide, on ? at_v : rows_v, on);
      }
    }
  }
  // the query row of column lane / 4 as it is read (null: none), and taken
  static constexpr int kRaw = DP / 8;
  static __device__ __forceinline__ void read(const CacheArgs& a, const uint8_t* row, uint32_t* x) {
    const int c = threadIdx.x % 4;
#pragma unroll
    for (int i = 0; i < kRaw; ++i) {
      const int d = 8 * i + 2 * c;
      x[i] = row && d < a.dim ? __ldg(reinterpret_cast<const uint32_t*>(row + 2 * d)) : 0;
    }
  }
  __device__ __forceinline__ void queries(const CacheArgs& a, int nt, const uint32_t* x) {
    f = a.scale * 1.4426950408889634f;
#pragma unroll
    for (int i = 0; i < kRaw; ++i) q[i / 2][nt][i % 2] = x[i];
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
  template <int T>
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
  __device__ __forceinline__ void outputs(uint32_t stage, int, const float (*p1)[NT][4]) {
    const int lane = threadIdx.x % 32, key = lane % 8 + lane / 16 * 8;
    const float(*p)[4] = p1[0];
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
  // put(entry, column 2 c + j, value) for all of this lane's outputs
  template <class F>
  __device__ __forceinline__ void each(int nt, F&& put) const {
    const int r = threadIdx.x % 32 / 4;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) put(16 * i + r + e / 2 * 8, e % 2, o[i][nt][e]);
  }
  // the outputs of column lane / 4, times its factor, to its row (null: none)
  __device__ __forceinline__ void store(const CacheArgs& a, int nt, const float* by, uint8_t* row) const {
    const int c = threadIdx.x % 4;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t x = transposed(pack2<BF16>(o[i][nt][2 * h] * by[0], o[i][nt][2 * h + 1] * by[1]));
        const int d = 16 * i + 8 * h + 2 * c;
        if (row && d < a.dim) *reinterpret_cast<uint32_t*>(row + 2 * d) = x;
      }
  }
};

template <int G, int NT, bool BF16>
struct Narrow {                            // 4 bits, G groups of 32 entries
  static constexpr int kBits = 4;
  static constexpr bool kPaged = true;
  // Two times 16 keys at once where there are registers for them: what is done
  // once per tile counts half, and one's instructions cover the other's.
  static constexpr int DP = 32 * G, MT = NT == 1 ? 2 : 1, kStages = MT == 2 ? 3 : 4, kSide = kKeys * 16 * G, kScales = kKeys * 2 * G;
  static constexpr int kPart = 2 * (kSide + kScales), kStage = MT * kPart;
  uint32_t q[2 * G][NT][2], start[NT][2];  // start: -8 sum q of each group, as sums of two float16
  float o[2 * G][NT][4];
  float f[NT][2];
  __half2 by[(G + 1) / 2];                 // 1 / bound of each group: a power of two that none of its scales so far reaches

  const uint8_t *k, *v, *scale;            // what the copies of 16 keys start from
  uint32_t to_v, to_scale;
  uint32_t at_k, at_v, at_scale;           // where this lane reads
  __device__ __forceinline__ void begin(const CacheArgs& a, uint32_t) {
    const int lane = threadIdx.x % 32, key = lane / G, j = lane % G, i = lane % (2 * G), r = lane / 4, c = lane % 4;
    k = a.k + 16 * lane;
    v = a.v + 16 * lane;
    // rows of values: even keys first, so that the four keys of a product's slots lie side by side
    to_v = kSide + (key / 2 + key % 2 * 8) * 16 * G + 16 * j;
    scale = (lane < 2 * G ? a.k_scale : a.v_scale) + 16 * i;
    to_scale = 2 * kSide + (lane < 2 * G ? 0 : kScales) + 16 * i;
    at_k = r * 16 * G + 4 * G * c;
    at_v = kSide + c * 16 * G + 4 * G * (r / 2);
    at_scale = 2 * kSide + r * 2 * G;
  }
  // (Rows past the sequence's end come too: codes are numbers whatever they are,
  // and outputs() leaves out their scales.)
  template <int T>
  __device__ __forceinline__ void fetch(const CacheArgs&, uint32_t stage, uint32_t row16, int) const {
    const int lane = threadIdx.x % 32;
    const uint8_t *from_k = k + (uint64_t)row16 * (256 * G), *from_v = v + (uint64_t)row16 * (256 * G);
    const uint32_t put_k = stage + 16 * lane, put_v = stage + to_v;
    unrolled<(kKeys * G + 31) / 32>([&](auto step) {
      constexpr int E = 32 * decltype(step)::value;
      if (E + 32 <= kKeys * G || lane < kKeys * G - E) {
        copy16<T * kPart + 16 * E, 16 * E>(put_k, from_k);
        if constexpr (32 % (2 * G) == 0) { // 32 pieces further is a whole, even number of keys further
          copy16<T * kPart + E / (2 * G) * 16 * G, 16 * E>(put_v, from_v);
        } else {
          const int key = (lane + E) / G, j = (lane + E) % G;
          copy16<T * kPart + kSide, 16 * E>(stage + (key / 2 + key % 2 * 8) * 16 * G + 16 * j, from_v);
        }
      }
    });
    if (lane < 4 * G) copy16<T * kPart, 0>(stage + to_scale, scale + (uint64_t)row16 * (32 * G));   // 2 G pieces for keys, then for values
  }
  static constexpr int kRaw = 4 * G;
  static __device__ __forceinline__ void read(const CacheArgs&, const uint8_t* row, uint32_t* x) {
    const int c = threadIdx.x % 4;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row) v = __ldg(reinterpret_cast<const uint4*>(row + 2 * (32 * w + 8 * c)));
      x[4 * w] = v.x;
      x[4 * w + 1] = v.y;
      x[4 * w + 2] = v.z;
      x[4 * w + 3] = v.w;
    }
  }
  __device__ __forceinline__ void queries(const CacheArgs& a, int nt, const uint32_t* raw) {
    const int c = threadIdx.x % 4;
    float x[G][8];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kRaw; ++i) {
      const float2 y = unpack2<BF16>(raw[i]);
      x[i / 4][2 * (i % 4)] = y.x;
      x[i / 4][2 * (i % 4) + 1] = y.y;
      top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
    }
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
    // the head's largest entry into 2^14 .. 2^15
    const int k = min(100, 14 + 127 - (int)(__float_as_uint(top) >> 23));
    const float up = __uint_as_float((uint32_t)(127 + k) << 23), down = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
    for (int w = 0; w < G; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        q[2 * w + h][nt][0] = pack2<false>(x[w][2 * h] * up, x[w][2 * h + 4] * up);
        q[2 * w + h][nt][1] = pack2<false>(x[w][2 * h + 1] * up * 0.0625f, x[w][2 * h + 5] * up * 0.0625f);
      }
#pragma unroll
    for (int j = 0; j < 2; ++j)            // (not 0, which would make a NaN of a hidden score, nor infinity: of a score of 0)
      f[nt][j] = fminf(fmaxf(a.scale * 1.4426950408889634f * 16777216.f * __shfl_sync(~0u, down, (2 * c + j) * 4), 1.17549435e-38f), 3.40282347e38f);
    // -8 sum q of the groups, to lanes c = 0 (groups 0, 1) and 1 (2, 3), and what
    // their rounding leaves to lanes c = 2 and 3
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < G; ++w) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 u = unpack2<false>(q[2 * w + h][nt][0]), t = unpack2<false>(q[2 * w + h][nt][1]);
        sum[w] += u.x + u.y + 16.f * (t.x + t.y);
      }
      sum[w] += __shfl_xor_sync(~0u, sum[w], 1);
      sum[w] += __shfl_xor_sync(~0u, sum[w], 2);
      sum[w] *= -8.f / 16777216.f;
    }
    float s0 = c % 2 ? sum[2] : sum[0], s1 = c % 2 ? sum[3] : sum[1];
    if (c >= 2) {
      const float2 t = unpack2<false>(pack2<false>(s0, s1));
      s0 -= t.x;
      s1 -= t.y;
    }
    start[nt][0] = pack2<false>(s0, s1);
    start[nt][1] = 0;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (G + 1) / 2; ++i) by[i] = as_half2(0x7c007c00u);   // (infinity)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) o[i][nt][e] = 0.f;
  }
  __device__ __forceinline__ float factor(int nt, int j) const { return f[nt][j]; }
  __device__ __forceinline__ float inverse(int w) const { return w % 2 ? __high2float(by[w / 2]) : __low2float(by[w / 2]); }
  // the scales of keys r and r + 8, as they lie: G halves each
  template <int AT>
  static __device__ __forceinline__ void scales(uint32_t at, uint32_t (*x)[(G + 1) / 2]) {
    if constexpr (G % 2 == 0) {
      read_words<G / 2, AT>(at, x[0]);
      read_words<G / 2, AT + 16 * G>(at, x[1]);
    } else {
      x[0][0] = read_half<AT>(at);
      x[1][0] = read_half<AT + 16 * G>(at);
      if constexpr (G == 3) {
        x[0][0] |= read_half<AT + 2>(at) << 16;
        x[1][0] |= read_half<AT + 2 + 16 * G>(at) << 16;
        x[0][1] = read_half<AT + 4>(at);
        x[1][1] = read_half<AT + 4 + 16 * G>(at);
      }
    }
  }
  template <int T>
  __device__ __forceinline__ void scores(uint32_t stage, float (*s)[4]) const {
    const int c = threadIdx.x % 4;
    uint32_t x[2][G], sc[2][(G + 1) / 2];
    read_words<G, T * kPart>(stage + at_k, x[0]);
    read_words<G, T * kPart + 8 * 16 * G>(stage + at_k, x[1]);
    scales<T * kPart>(stage + at_scale, sc);
    // the sums' start: scales by -8 sum q
    const bool odd = c % 2;
    const uint32_t both[4] = {G > 2 && odd ? sc[0][(G + 1) / 2 - 1] : odd ? 0 : sc[0][0], G > 2 && odd ? sc[1][(G + 1) / 2 - 1] : odd ? 0 : sc[1][0], 0, 0};
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mma<false>(s[nt], both, start[nt][0], start[nt][1], zero);
#pragma unroll
    for (int w = 0; w < G; ++w) {
      const uint32_t lo[4] = {x[0][w] & 0x000f000fu, x[1][w] & 0x000f000fu, x[0][w] & 0x00f000f0u, x[1][w] & 0x00f000f0u};
      const uint32_t y0 = x[0][w] >> 8, y1 = x[1][w] >> 8;
      const uint32_t hi[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
      const float2 k0 = __half22float2(as_half2(sc[0][w / 2])), k1 = __half22float2(as_half2(sc[1][w / 2]));
      const float u0 = w % 2 ? k0.y : k0.x, u1 = w % 2 ? k1.y : k1.x;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float d[4];
        mma<false>(d, lo, q[2 * w][nt][0], q[2 * w][nt][1], zero);
        mma<false>(d, hi, q[2 * w + 1][nt][0], q[2 * w + 1][nt][1], d);
        s[nt][0] = fmaf(u0, d[0], s[nt][0]);
        s[nt][1] = fmaf(u0, d[1], s[nt][1]);
        s[nt][2] = fmaf(u1, d[2], s[nt][2]);
        s[nt][3] = fmaf(u1, d[3], s[nt][3]);
      }
    }
  }
  __device__ __forceinline__ void outputs(uint32_t stage, int keys, const float (*p)[NT][4]) {
    const int r = threadIdx.x % 32 / 4;
    uint32_t sc[MT][2][(G + 1) / 2];
    unrolled<MT>([&](auto t) { scales<decltype(t)::value * kPart + kScales>(stage + at_scale, sc[decltype(t)::value]); });
    if (keys < MT * kKeys) {               // past the sequence's end a scale may be anything, and a zero weight does not hide a NaN
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < (G + 1) / 2; ++i) sc[t][e][i] = 16 * t + r + 8 * e < keys ? sc[t][e][i] : 0;
    }
    __half2 most[(G + 1) / 2];
    bool larger = false;                                     // than any scale of its group so far (or the first tile)
#pragma unroll
    for (int i = 0; i < (G + 1) / 2; ++i) {
      most[i] = __hmax2(as_half2(sc[0][0][i]), as_half2(sc[0][1][i]));
#pragma unroll
      for (int t = 1; t < MT; ++t) most[i] = __hmax2(most[i], __hmax2(as_half2(sc[t][0][i]), as_half2(sc[t][1][i])));
      larger = larger || __hgeu2_mask(__hmul2(most[i], by[i]), as_half2(0x3c003c00u)) != 0;
    }
    if (__any_sync(~0u, larger)) {
#pragma unroll
      for (int i = 0; i < (G + 1) / 2; ++i) {
#pragma unroll
        for (int e = 4; e < 32; e *= 2) most[i] = __hmax2(most[i], as_half2(__shfl_xor_sync(~0u, as_word(most[i]), e)));
        const float2 top = __half22float2(most[i]), was = __half22float2(by[i]);
        float now[2] = {1.f, 1.f};
#pragma unroll
        for (int h = 0; h < 2 && 2 * i + h < G; ++h) {
          const int w = 2 * i + h;
          // the power of two above it, 2^-13 to 2^16
          const uint32_t above = min(max(__float_as_uint(h ? top.y : top.x) >> 23, 127u - 14u), 127u + 15u) + 1;
          now[h] = fminf(h ? was.y : was.x, __uint_as_float((254u - above) << 23));
          const float ratio = now[h] / (h ? was.y : was.x);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              o[2 * w][nt][e] *= ratio;
              o[2 * w + 1][nt][e] *= ratio;
            }
        }
        by[i] = __floats2half2_rn(now[0], now[1]);
      }
    }
    const uint32_t halves = r % 2 ? 0x7632u : 0x5410u;
    const uint32_t eight[4] = {0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u};   // -8, and 16 times that
    unrolled<MT>([&](auto part) {
      constexpr int T = decltype(part)::value;
      __half2 rel[2][(G + 1) / 2], h[NT][2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < (G + 1) / 2; ++i) rel[e][i] = __hmul2(as_half2(sc[T][e][i]), by[i]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        h[nt][0] = as_half2(pack2<false>(p[T][nt][0], p[T][nt][1]));
        h[nt][1] = as_half2(pack2<false>(p[T][nt][2], p[T][nt][3]));
      }
      uint32_t x[4][G];                                      // keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
      unrolled<4>([&](auto key) {
        constexpr int E = decltype(key)::value;
        read_words<G, T * kPart + (E / 2 * 4 + E % 2 * 8) * 16 * G>(stage + at_v, x[E]);
      });
#pragma unroll
      for (int w = 0; w < G; ++w) {
        uint32_t b[NT][2];
        const __half2 r0 = w % 2 ? __high2half2(rel[0][w / 2]) : __low2half2(rel[0][w / 2]);
        const __half2 r1 = w % 2 ? __high2half2(rel[1][w / 2]) : __low2half2(rel[1][w / 2]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          b[nt][0] = transposed(as_word(__hmul2(h[nt][0], r0)));
          b[nt][1] = transposed(as_word(__hmul2(h[nt][1], r1)));
        }
        const uint32_t y0 = __byte_perm(x[0][w], x[1][w], halves), y1 = __byte_perm(x[2][w], x[3][w], halves);
        const uint32_t lo[4] = {y0 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x000f000fu, y1 & 0x00f000f0u};
        const uint32_t z0 = y0 >> 8, z1 = y1 >> 8;
        const uint32_t hi[4] = {z0 & 0x000f000fu, z0 & 0x00f000f0u, z1 & 0x000f000fu, z1 & 0x00f000f0u};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma<false>(o[2 * w][nt], lo, b[nt][0], b[nt][1], o[2 * w][nt]);
          mma<false>(o[2 * w + 1][nt], hi, b[nt][0], b[nt][1], o[2 * w + 1][nt]);
          mma<false>(o[2 * w][nt], eight, b[nt][0], b[nt][1], o[2 * w][nt]);
          mma<false>(o[2 * w + 1][nt], eight, b[nt][0], b[nt][1], o[2 * w + 1][nt]);
        }
      }
    });
  }
  __device__ __forceinline__ void rescale(int nt, int j, float by_) {
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
      o[i][nt][j] *= by_;
      o[i][nt][j + 2] *= by_;
    }
  }
  // output entries 32 w + 4 r + 2 h (s = 0) and the one after it (s = 1) of column 2 c + j
  __device__ __forceinline__ float output(int w, int h, int s, int nt, int j) const {
    return o[2 * w + h][nt][j + 2 * s] * ((s ? 1048576.f : 16777216.f) * __frcp_rn(inverse(w)));
  }
  template <class F>
  __device__ __forceinline__ void each(int nt, F&& put) const {
    const int r = threadIdx.x % 32 / 4;
#pragma unroll
    for (int w = 0; w < G; ++w)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 2; ++s) put(32 * w + 4 * r + 2 * h + s, j, output(w, h, s, nt, j));
  }
  __device__ __forceinline__ void store(const CacheArgs&, int nt, const float* by, uint8_t* row) const {
    const int c = threadIdx.x % 4;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      uint32_t x[2][2];                    // entries 8 c + 2 h + s and 8 c + 4 + 2 h + s of column r
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          x[h][s] = transposed(pack2<BF16>(output(w, h, s, nt, 0) * by[0], output(w, h, s, nt, 1) * by[1]));
      if (row)
        *reinterpret_cast<uint4*>(row + 2 * (32 * w + 8 * c)) =
            make_uint4(__byte_perm(x[0][0], x[0][1], 0x5410), __byte_perm(x[1][0], x[1][1], 0x5410),
                       __byte_perm(x[0][0], x[0][1], 0x7632), __byte_perm(x[1][0], x[1][1], 0x7632));
    }
  }
};

// ---- division of the work ----
template <bool PAGED>
__device__ __forceinline__ Shape shape_of(const CacheArgs& a, int s, int rows, int tile) {
  const int64_t begin = a.starts ? __ldg(a.starts + s) : s;
  const int64_t end = !PAGED ? begin + __ldg(a.counts + s) : a.starts ? __ldg(a.starts + s + 1) : s + 1;
  return division::shape(begin, end, a.rows, __ldg(a.lens + s), PAGED ? a.max_pages << a.page_shift : INT32_MAX, a.heads / a.kv_heads, a.kv_heads, rows, tile, a.whole);
}

// (A call of its own: in line it takes the calls that never need it half a
// microsecond of ten.)
__device__ __noinline__ int behind_empty(const int32_t* starts, int s, int n_seqs) {
  return division::behind_empty([&](int i) { return __ldg(starts + i); }, s, n_seqs);
}

// The runs of a block's warps: their bounds in the list, and the sequences where
// they begin with how far into them.
struct Runs {
  int64_t sum[kWarps], bound[kWarps + 1], into[kWarps], total;
  int s[kWarps], takers;
  Shape shape[kWarps];                     // of that sequence
};

__device__ __forceinline__ int64_t summed_up(int64_t x) {     // over the lanes up to this one
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int64_t up = __shfl_up_sync(~0u, x, o);
    if (threadIdx.x % 32 >= o) x += up;
  }
  return x;
}

template <int ROWS, int TILE, bool PAGED>
__device__ __forceinline__ void find_runs(const CacheArgs& a, Runs& runs) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const bool few = a.n_seqs <= kThreads;
  int64_t cost = 0;
  Shape x{};
  for (int s = threadIdx.x; s < a.n_seqs; s += kThreads) {
    x = shape_of<PAGED>(a, s, ROWS, TILE);
    cost += x.cost;
  }
  int64_t sum = summed_up(cost);
  if (lane == 31) runs.sum[warp] = sum;
  __syncthreads();
  if (threadIdx.x <= kWarps) {
    const int64_t total = runs.sum[0] + runs.sum[1] + runs.sum[2] + runs.sum[3];
    const int takers = division::takers(total, gridDim.x * kWarps, a.whole);
    runs.bound[threadIdx.x] = division::bound(total, takers, blockIdx.x * kWarps + threadIdx.x);
    if (threadIdx.x == 0) {
      runs.total = total;
      runs.takers = takers;
    }
  }
  __syncthreads();
  if (runs.bound[0] == runs.bound[kWarps]) return;
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kThreads) {
    const int s = s0 + threadIdx.x;
    if (!few) {
      if (s < a.n_seqs) x = shape_of<PAGED>(a, s, ROWS, TILE);
      cost = s < a.n_seqs ? x.cost : 0;
      sum = summed_up(cost);
      __syncthreads();
      if (lane == 31) runs.sum[warp] = sum;
      __syncthreads();
    }
    int64_t mine = before + sum - cost;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) mine += runs.sum[w];
      before += runs.sum[w];
    }
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int64_t at = runs.bound[w];
      if (at < runs.bound[w + 1] && mine <= at && at < mine + cost) {
        runs.s[w] = s;
        runs.into[w] = at - mine;
        runs.shape[w] = x;
      }
    }
    if (before > runs.bound[kWarps - 1]) break;
  }
  __syncthreads();
}

// N entries of a piece's row, a multiple of N from its start, in wide accesses.
template <int N>
struct Entries {
  static constexpr int kVec = N % 4 == 0 ? 4 : 2;
  static __device__ __forceinline__ void load(const float* p, float* x) {
#pragma unroll
    for (int e = 0; e < N; e += kVec) {
      if constexpr (kVec == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + e);
        x[e] = v.x;
        x[e + 1] = v.y;
        x[e + 2] = v.z;
        x[e + 3] = v.w;
      } else {
        const float2 v = *reinterpret_cast<const float2*>(p + e);
        x[e] = v.x;
        x[e + 1] = v.y;
      }
    }
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
#pragma unroll
    for (int e = 0; e < N; e += kVec) {
      if constexpr (kVec == 4) *reinterpret_cast<float4*>(p + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      else *reinterpret_cast<float2*>(p + e) = make_float2(x[e], x[e + 1]);
    }
  }
};

// DP / 16 entries of an output row from d0 on, from their sums with weights of
// maximum `top` and sum `sum`.
template <int DP, bool BF16>
__device__ __forceinline__ void finish_row(const CacheArgs& a, int64_t row, int head, int d0, const float* acc, float top, float sum) {
  uint8_t* const to = static_cast<uint8_t*>(a.q_out.data) + 2 * (row * a.q_out.row + head * a.q_out.head);
  const float by = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < DP / 16; e += 2)
    if (d0 + e < a.dim) *reinterpret_cast<uint32_t*>(to + 2 * (d0 + e)) = pack2<BF16>(acc[e] * by, acc[e + 1] * by);
  if (a.lse && d0 == 0) a.lse[head * a.rows + row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

// What a warp leaves of passes that it did not do alone: the end of one that
// began before (its rows are in the workspace), and one that it did not end (in
// the warp's shared memory).
struct Left {
  int before;
  int open;                                // 1: that it began; 2: that began before
  int row0[2], n[2], head[2], first[2];    // of either, as in Piece
  int last;                                // of the open one: the block that ends it
};

template <class K, int NT, bool BF16>
__global__ void __launch_bounds__(kThreads, per_sm(K::kBits, NT)) k_cache_attn(const __grid_constant__ CacheArgs a) {
  constexpr int DP = K::DP, MT = K::MT, ROWS = 8 * NT, S = K::kStages, kTile = MT * kKeys, kRing = S * K::kStage;
  using P = Parts<DP, ROWS>;
  static_assert(P::kFloats * 4 <= kRing, "a warp's shared memory holds a pass");
  // (aligned: a copy of 32 bytes by two lanes to halves of two such pieces reads them twice from L2)
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ Piece lists[kWarps][kPieces];
  __shared__ Lister listers[kWarps];
  __shared__ Left lefts[kWarps];
  __shared__ Runs runs;
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
  const int group = a.heads / a.kv_heads;
  const uint32_t mine = smem_addr(ring) + warp * kRing;
  float* const parts = reinterpret_cast<float*>(a.work + P::header(gridDim.x));
  auto out_row = [&](const int64_t row, int head) { return static_cast<uint8_t*>(a.q_out.data) + 2 * (row * a.q_out.row + head * a.q_out.head); };

  if (a.fill) {                            // padding in front of the first sequence and behind the last
    auto start = [&](int s) { return min(max((int64_t)__ldg(a.starts + s), (int64_t)0), a.rows); };
    const int64_t first = a.starts ? start(0) : 0, end = a.starts ? max(first, start(a.n_seqs)) : a.rows;
    for (int64_t pad = blockIdx.x; pad < first + a.rows - end; pad += gridDim.x) {
      const int64_t row = pad < first ? pad : end + pad - first;
      for (int i = threadIdx.x; i < a.heads * (a.dim / 8); i += kThreads) {
        const int h = i / (a.dim / 8), d = i % (a.dim / 8) * 8;
        *reinterpret_cast<uint4*>(out_row(row, h) + 2 * d) = make_uint4(0, 0, 0, 0);
        if (a.lse && d == 0) a.lse[h * a.rows + row] = -INFINITY;
      }
    }
  }

  find_runs<ROWS, kTile, K::kPaged>(a, runs);
  Lister& lister = listers[warp];
  Piece* const list = lists[warp];
  Left& left = lefts[warp];
  if (lane == 0) {
    left.before = left.open = 0;
    lister.left = runs.bound[warp + 1] - runs.bound[warp];
    if (lister.left) lister.start(runs.shape[warp], runs.s[warp], runs.bound[warp], runs.into[warp], lister.left);
  }
  K k;
  k.begin(a, mine);

  // The next piece of this warp, in a ring of kPieces (the copies are at most S
  // tiles, and so pieces, ahead).  Passes without keys are done here.
  auto after_empty = [&](int s) {
    return K::kPaged && a.starts ? behind_empty(a.starts, s, a.n_seqs) : s + 1;
  };
  int made = 0;
  bool done = false;
  auto make = [&] {
    for (;;) {
      if (done) return false;
      int ok = 0;
      if (lane == 0) ok = lister.next([&](int s) { return shape_of<K::kPaged>(a, s, ROWS, kTile); }, after_empty, a.n_seqs, a.kv_heads, ROWS, a.whole, list[made % kPieces]);
      __syncwarp();
      done = !__shfl_sync(~0u, ok, 0);
      if (done) return false;
      const Piece& x = list[made % kPieces];
      if (x.from < x.to) {
        ++made;
        return true;
      }
      const uint32_t fill = x.bad ? 0x7fff7fffu : 0u;        // NaN in both types
      for (int i = lane; i < ROWS * (a.dim / 8); i += 32) {
        const int row = x.first + i / (a.dim / 8), d = i % (a.dim / 8) * 8, head = x.head * group + row % group;
        if (row >= x.n * group) break;
        *reinterpret_cast<uint4*>(out_row(x.row0 + row / group, head) + 2 * d) = make_uint4(fill, fill, fill, fill);
        if (a.lse && d == 0) a.lse[head * a.rows + x.row0 + row / group] = x.bad ? __int_as_float(0x7fffffff) : -INFINITY;
      }
      __syncwarp();
    }
  };

  // Tiles ahead: the next one to copy, whose page was looked up one tile before.
  int ap = 0, at_tile = 0, at_to = 0, at_len = 0, at_head = 0, page[MT];
  const int32_t* at_table = nullptr;
  const uint8_t *at_k = nullptr, *at_v = nullptr;   // plain rows: the sequence's first key and value
  auto piece = [&] {                       // at_len 0 behind the last
    at_len = 0;
    if (ap == made && !make()) return;
    const Piece& x = list[ap++ % kPieces];
    at_tile = x.from;
    at_to = x.to;
    at_len = x.len;
    at_head = x.head;
    if constexpr (K::kPaged) {
      at_table = a.table + x.s * a.table_stride;
    } else {
      const int64_t row = __ldg(a.firsts + x.s);
      at_k = static_cast<const uint8_t*>(a.k_rows.data) + 2 * (row * a.k_rows.row + at_head * a.k_rows.head);
      at_v = static_cast<const uint8_t*>(a.v_rows.data) + 2 * (row * a.v_rows.row + at_head * a.v_rows.head);
    }
  };
  auto look = [&] {
    if (!K::kPaged) return;
    const int pos = at_tile * kTile;
    if (at_len) page[0] = __ldg(at_table + (pos >> a.page_shift));
    if (MT == 2 && a.page_shift == 4 && pos + kKeys < at_len) page[MT - 1] = __ldg(at_table + (pos >> a.page_shift) + 1);
  };
  uint32_t put = mine, lost = 0;           // lost: stages whose page the cache does not have
  auto ahead = [&] {
    if (at_len) {
      const int pos = at_tile * kTile;
      if constexpr (K::kPaged) {
        auto row16 = [&](int t) {
          return (((uint32_t)page[t] * a.kv_heads + at_head) << (a.page_shift - 4)) + (pos / kKeys & ((1 << (a.page_shift - 4)) - 1));
        };
        const bool two = MT == 2 && pos + kKeys < at_len, apart = a.page_shift == 4;
        bool has = (unsigned)page[0] < (unsigned)a.n_pages;
        const uint32_t first = row16(0);
        if (has) k.template fetch<0>(a, put, first, at_len - pos);
        if (two && apart) {
          has = has && (unsigned)page[MT - 1] < (unsigned)a.n_pages;
          if (has) k.template fetch<MT - 1>(a, put, row16(MT - 1), at_len - pos - kKeys);
        } else if (two && has) {
          k.template fetch<MT - 1>(a, put, first + 1, at_len - pos - kKeys);
        }
        if (!has) lost |= 1u << (put - mine) / K::kStage;
      } else {
        k.copy(a, put, at_k + pos * k.k_step, at_v + pos * k.v_step, at_len - pos);
      }
      if (++at_tile >= at_to) piece();
      look();
    }
    end_group();
    put = put + K::kStage == mine + kRing ? mine : put + K::kStage;
  };
  piece();
  look();
  __syncwarp();
#pragma unroll 1
  for (int i = 0; i < S - 1; ++i) ahead();
  uint32_t get = mine;

  // the query of a column: head and token of a row of the pass
  auto split = [&](const Piece& x, int row, int& token, int& head) {
    token = x.n == 1 ? 0 : row / group;
    head = x.head * group + (x.n == 1 ? row : row - token * group);
  };
  auto query = [&](const Piece& x, int nt) -> const uint8_t* {
    const int row = x.first + 8 * nt + r;
    int token, head;
    split(x, row, token, head);
    return row < x.n * group ? static_cast<const uint8_t*>(a.q.data) + 2 * ((x.row0 + token) * a.q.row + head * a.q.head) : nullptr;
  };
  uint32_t raw[K::kRaw];                   // the next piece's queries, where there are registers for them
  if (NT == 1 && made) K::read(a, query(list[0], 0), raw);
  // (the copies, a tile ahead at least, have asked for the next piece before one is done)
#pragma unroll 1
  for (int ip = 0; ip < made; ++ip) {
    const Piece& x = list[ip % kPieces];
    const int len = x.len, to = x.to;
    float m[NT][2], l[NT][2], shift[NT][2];   // shift: what weights are relative to, m less kLift; 0 where nothing was seen
    int limit[NT][2];                      // tokens that a column's row sees
    int least = len;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (NT > 1) K::read(a, query(x, nt), raw);
      k.queries(a, nt, raw);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        int token, head;
        split(x, x.first + 8 * nt + 2 * c + j, token, head);
        m[nt][j] = -INFINITY;
        l[nt][j] = shift[nt][j] = 0.f;
        limit[nt][j] = K::kPaged ? len - x.n + min(token, x.n - 1) + 1 : len;
        least = min(least, limit[nt][j]);
      }
    }
    k.clear();
    bool bad = x.bad;
    // from this token on some row does not see a tile whole
    const int whole_to = __all_sync(~0u, least == len) ? len - kTile : -1;
#pragma unroll 1
    for (int tile = x.from; tile < to; ++tile) {
      __syncwarp();
      ahead();
      wait_groups<S - 1>();
      __syncwarp();
      const uint32_t stage = get;
      const int pos = tile * kTile;
      get = get + K::kStage == mine + kRing ? mine : get + K::kStage;
      if (lost) {
        const uint32_t bit = 1u << (stage - mine) / K::kStage;
        if (lost & bit) {
          lost &= ~bit;
          bad = true;
          continue;
        }
      }
      float s[MT][NT][4];
      unrolled<MT>([&](auto t) { k.template scores<decltype(t)::value>(stage, s[decltype(t)::value]); });
      if (pos > whole_to) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[t][nt][e] = pos + kKeys * t + r + e / 2 * 8 < limit[nt][e % 2] ? s[t][nt][e] : -INFINITY;
      }
      float top[NT][2];
      bool rises = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          top[nt][j] = fmaxf(s[0][nt][j], s[0][nt][j + 2]);
#pragma unroll
          for (int t = 1; t < MT; ++t) top[nt][j] = fmaxf(top[nt][j], fmaxf(s[t][nt][j], s[t][nt][j + 2]));
          top[nt][j] *= k.factor(nt, j);
          rises = rises || top[nt][j] > m[nt][j] + kLag;
        }
      if (__any_sync(~0u, rises)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int o = 4; o < 32; o *= 2) top[nt][j] = fmaxf(top[nt][j], __shfl_xor_sync(~0u, top[nt][j], o));
            if (top[nt][j] > m[nt][j] + kLag) {
              const float to = top[nt][j] - (fabsf(top[nt][j]) < kSure ? kLift : 0.f);
              const float by = m[nt][j] == -INFINITY ? 0.f : exp2_fast(shift[nt][j] - to);
              m[nt][j] = top[nt][j];
              shift[nt][j] = to;
              l[nt][j] *= by;
              k.rescale(nt, j, by);
            }
          }
      }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[t][nt][e] = exp2_fast(fmaf(s[t][nt][e], k.factor(nt, e % 2), -shift[nt][e % 2]));
            l[nt][e % 2] += s[t][nt][e];
          }
      k.outputs(stage, len - pos, s);
    }
    if (NT == 1 && ip + 1 < made) K::read(a, query(list[(ip + 1) % kPieces], 0), raw);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int o = 4; o < 32; o *= 2) l[nt][j] += __shfl_xor_sync(~0u, l[nt][j], o);
        if (bad) l[nt][j] = __int_as_float(0x7fffffff);
      }
    if (x.from == 0 && to == x.tiles) {    // all of the pass
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float by[2] = {l[nt][0] == 0.f ? 0.f : 1.f / l[nt][0], l[nt][1] == 0.f ? 0.f : 1.f / l[nt][1]};
        const int row = x.first + 8 * nt + r;
        int token, head;
        split(x, row, token, head);
        k.store(a, nt, by, row < x.n * group ? out_row(x.row0 + token, head) : nullptr);
        if (a.lse && r == 0)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            split(x, x.first + 8 * nt + 2 * c + j, token, head);
            if (x.first + 8 * nt + 2 * c + j < x.n * group)
              a.lse[head * a.rows + x.row0 + token] = l[nt][j] == 0.f ? -INFINITY : (shift[nt][j] + log2f(l[nt][j])) * 0.6931471805599453f;
          }
      }
    } else {
      const int open = to < x.tiles;       // the warp's last piece: its shared memory is free
      float* const part = open ? reinterpret_cast<float*>(ring + warp * kRing) : parts + P::warp_slot(gridDim.x, blockIdx.x * kWarps + warp);
      if (open) {
        wait_groups<0>();
        __syncwarp();
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        k.each(nt, [&](int d, int j, float v) { part[(8 * nt + 2 * c + j) * P::kRow + d] = v; });
        if (r == 0)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            part[(8 * nt + 2 * c + j) * P::kRow + DP] = m[nt][j] == -INFINITY ? -INFINITY : shift[nt][j];
            part[(8 * nt + 2 * c + j) * P::kRow + DP + 1] = l[nt][j];
          }
      }
      if (lane == 0) {
        if (open) left.open = x.from ? 2 : 1;
        else left.before = 1;
        left.row0[open] = x.row0;
        left.n[open] = x.n;
        left.head[open] = x.head;
        left.first[open] = x.first;
        if (open) left.last = division::holder(runs.total, runs.takers, x.last_tile()) / kWarps;
      }
    }
    __syncwarp();
  }
  wait_groups<0>();
  if (a.whole) return;
  __syncthreads();

  // Passes of which several warps have pieces, in the order of the warps: a chain
  // from a warp's open pass over those that it goes on in to one that ends it.
  // What is still open at either end of the block goes to the second kernel.
  constexpr int kEach = DP / 16;
  Header header{0, 0, 0, 0, 0, 0};
  auto join = [&](int a0, int b, bool ended, bool led) {
    const Left& of = lefts[ended ? b : a0];
    const int which = ended ? 0 : 1, row0 = of.row0[which], n = of.n[which], head = of.head[which], first = of.first[which];
    const bool whole = ended && !led;
    const int slot = 2 * blockIdx.x + (ended || led ? 0 : 1);
    if (!led && !ended) header = Header{1, of.last, row0, n, head, first};
    // 16 threads a row, for all rows at once: what they wait for is one read of
    // the pieces' maxima and one of their entries
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 8 * nt + threadIdx.x / 16, d0 = threadIdx.x % 16 * kEach;
      if (first + row >= n * group) continue;
      const float* p[kWarps + 1];
      float m[kWarps + 1], l[kWarps + 1], top = -INFINITY, sum = 0.f, acc[kEach];
#pragma unroll
      for (int w = 0; w <= kWarps; ++w) {
        p[w] = w < kWarps ? (w >= a0 && w < b ? reinterpret_cast<const float*>(ring + w * kRing) + row * P::kRow : nullptr)
                          : ended ? parts + P::warp_slot(gridDim.x, blockIdx.x * kWarps + b) + row * P::kRow : nullptr;
        m[w] = p[w] ? p[w][DP] : -INFINITY;
        l[w] = p[w] ? p[w][DP + 1] : 0.f;
        top = fmaxf(top, m[w]);
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w <= kWarps; ++w)
        if (p[w]) {
          const float f = m[w] == -INFINITY ? 0.f : exp2_fast(m[w] - top);
          sum += m[w] == -INFINITY ? l[w] : l[w] * f;         // (l is 0 or NaN where nothing was seen)
          float v[kEach];
          Entries<kEach>::load(p[w] + d0, v);
#pragma unroll
          for (int e = 0; e < kEach; ++e) acc[e] = fmaf(f, v[e], acc[e]);
        }
      if (whole) {
        const int token = (first + row) / group, h = head * group + (first + row) % group;
        finish_row<DP, BF16>(a, row0 + token, h, d0, acc, top, sum);
      } else {
        float* to = parts + P::slot(slot) + row * P::kRow;
        Entries<kEach>::store(to + d0, acc);
        if (d0 == 0) {
          to[DP] = top;
          to[DP + 1] = sum;
        }
      }
    }
  };
  bool going = false, led = false;
  int a0 = 0, last = 0;
#pragma unroll 1
  for (int w = 0; w < kWarps; ++w) {
    if (lefts[w].before) {
      join(going ? a0 : w, w, true, going ? led : true);
      going = false;
    }
    if (lefts[w].open) {
      if (!going) {
        a0 = w;
        led = lefts[w].open == 2;
      }
      going = true;
      last = w;
    }
  }
  if (going) join(a0, last + 1, false, led);
  if (threadIdx.x == 0) reinterpret_cast<Header*>(a.work)[blockIdx.x] = header;
}

// Passes that several blocks have pieces of, from these in order: a block for
// each block of the first kernel, if it began such a pass, and each of its rows;
// 16 threads on pieces in turn.  (Small blocks, which find room beside the first
// kernel's and wait there: of 512 threads they cost 5 us more.)
constexpr int kMergers = 8, kAtOnce = 3;
template <int DP, int ROWS, bool BF16>
__global__ void __launch_bounds__(16 * kMergers) k_cache_merge(const __grid_constant__ CacheArgs a, int blocks) {
  using P = Parts<DP, ROWS>;
  constexpr int kEach = DP / 16;
  __shared__ __align__(16) float sums[kMergers][DP + 4];
  after_previous();
  const Header* const headers = reinterpret_cast<const Header*>(a.work);
  const Header x = headers[blockIdx.x];
  const int group = a.heads / a.kv_heads, row = x.first + (int)blockIdx.y;
  if (!x.open || row >= x.n * group) return;
  const int mine = threadIdx.x / 16, l16 = threadIdx.x % 16, d0 = l16 * kEach;
  const float* const parts = reinterpret_cast<const float*>(a.work + P::header(blocks)) + blockIdx.y * P::kRow;
  auto part = [&](int b) { return parts + P::slot(2 * b + (b == (int)blockIdx.x)); };
  // this thread's pieces with the maximum so far: all reads of a few pieces at once
  float acc[kEach], sum = 0.f, top = -INFINITY;
#pragma unroll
  for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int b0 = blockIdx.x + mine; b0 <= x.last; b0 += kMergers * kAtOnce) {
    float m[kAtOnce], l[kAtOnce], v[kAtOnce][kEach], now = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int b = b0 + i * kMergers;
      m[i] = -INFINITY;
      l[i] = 0.f;
      if (b > x.last) continue;
      const float* p = part(b);
      m[i] = p[DP];
      l[i] = p[DP + 1];
      Entries<kEach>::load(p + d0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) now = fmaxf(now, m[i]);
    const float f = top == -INFINITY ? 0.f : exp2_fast(top - now);
    top = now;
    sum *= f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] *= f;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (b0 + i * kMergers > x.last) continue;
      const float g = m[i] == -INFINITY ? 0.f : exp2_fast(m[i] - top);
      sum += m[i] == -INFINITY ? l[i] : l[i] * g;           // (l is 0 or NaN where nothing was seen)
#pragma unroll
      for (int e = 0; e < kEach; ++e) acc[e] = fmaf(g, v[i][e], acc[e]);
    }
  }
  Entries<kEach>::store(&sums[mine][d0], acc);
  if (l16 == 0) {
    sums[mine][DP] = top;
    sums[mine][DP + 1] = sum;
  }
  __syncthreads();
  if (mine) return;
  top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kMergers; ++i) top = fmaxf(top, sums[i][DP]);
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kMergers; ++i) {
    const float m = sums[i][DP], l = sums[i][DP + 1], f = m == -INFINITY ? 0.f : exp2_fast(m - top);
    float v[kEach];
    Entries<kEach>::load(&sums[i][d0], v);
    sum += m == -INFINITY ? l : l * f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] = fmaf(f, v[e], acc[e]);
  }
  finish_row<DP, BF16>(a, x.row0 + row / group, x.head * group + row % group, d0, acc, top, sum);
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
  if (a.whole) return cudaSuccess;
  e = launch_early(k_cache_merge<K::DP, 8 * NT, BF16>, dim3((unsigned)a.blocks, 8 * NT), 16 * kMergers, 0, st, a, a.blocks);
  if (e == cudaSuccess) count_launch();
  return e;
}

template <int NT, bool BF16>
cudaError_t launch_rows(const CacheArgs& a, cudaStream_t st) {
  if (a.bits == 16) return a.dim <= 64 ? launch<Wide<64, NT, BF16, true>, NT, BF16>(a, st) : launch<Wide<128, NT, BF16, true>, NT, BF16>(a, st);
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

cudaError_t launch_few_queries(const CacheArgs& a, cudaStream_t st) {
  auto go = [&](auto bf16) {
    constexpr bool B = decltype(bf16)::value;
    if (a.most_rows == 16) return launch<Wide<64, 2, B, false>, 2, B>(a, st);   // (heads of up to 64 alone)
    return a.dim <= 64 ? launch<Wide<64, 1, B, false>, 1, B>(a, st) : launch<Wide<128, 1, B, false>, 1, B>(a, st);
  };
  return a.bf16 ? go(std::true_type()) : go(std::false_type());
}

int cache_attn_rows(int bits, int group, int max_new) {
  const int64_t rows = (int64_t)group * max_new;
  return rows <= 8 ? 8 : rows <= 16 || bits == 4 ? 16 : 32;
}

int cache_attn_blocks(int bits, int most_rows, int num_sms) { return per_sm(bits, most_rows / 8) * num_sms; }

int64_t cache_attn_workspace(int dim, int most_rows, int blocks) {
  const int dp = dim <= 64 ? 64 : 128;
  const size_t header = Parts<128, 32>::header(blocks);
  return (int64_t)(header + (size_t)Parts<128, 32>::kSlots * blocks * most_rows * (dp + 4) * sizeof(float));
}

cudaError_t launch_cache_attn(const CacheArgs& a, cudaStream_t st) {
  return a.bf16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace syncgb

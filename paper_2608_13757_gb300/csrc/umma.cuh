// sm_103a building blocks of the attention kernels: mbarriers whose waits
// give up, TMA tile loads, tcgen05 products with operands in shared memory
// or tensor memory, and tensor memory transfers.
//
// Tiles in shared memory are 128 rows of 64 16-bit entries (128 bytes a row)
// in the 128-byte swizzle that the TMA load writes, 16 KB each; wider rows
// take one such block per 64 entries.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace syncgb {
namespace umma {

// Lets a kernel take `bytes` of dynamic shared memory, once per device.
template <class K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (device & 63);
  if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

constexpr int kBlockBytes = 128 * 128;   // 128 rows of 64 entries

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(one));
  return one;
}

// ---- mbarriers ----
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_visible() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok;
}
// A wait by a whole warp, with one answer for all lanes.  One that never ends
// would be a defect: it gives up after kTries, about a second (the hardware
// suspends a try for 4 us), and says so in *error (host-visible).  A warp that
// gave up does nothing more, so the waits that depend on it give up too, and
// the kernel always ends.  (The longest wait of a sound call is that of a warp
// of the forward pass for an item of the other query tile, 0.8 us per 128 keys:
// a second for 160 million of them.)
//
// The kernels' code has to stay small: at 44 KB a change that added 8 KB
// outside all loops made the attention of a long prompt 15% slower, for the
// instruction cache.  So this is a short loop, and what is rare is a loop
// rather than unrolled.
constexpr int kTries = 1 << 18;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, int* error, int tries = kTries) {
#pragma unroll 1
  for (int i = 0; i < tries; ++i)
    if (__all_sync(~0u, bar_try(bar, parity))) return true;
  *reinterpret_cast<volatile int*>(error) = 1;
  return false;
}
// (What a warp decides, it decides by votes and by values of its first lane,
// which the compiler knows to be the same for all lanes: branches that may
// diverge cost more.)
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }
// One lane of the warp arrives, for all.
__device__ __forceinline__ void bar_arrive_warp(uint32_t bar, bool leader) {
  __syncwarp();
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %1, 0;\n@p mbarrier.arrive.shared::cta.b64 _, [%0];\n}" ::"r"(bar),
               "r"((uint32_t)leader)
               : "memory");
}

// The swizzle goes by address bits: tiles start at multiples of 1024 bytes, as
// the start of a block's shared memory does.
__device__ __forceinline__ bool swizzle_aligned(uint32_t base, int* error) {
  if (base % 1024 == 0) return true;
  if (threadIdx.x == 0) *reinterpret_cast<volatile int*>(error) = 1;
  return false;
}

// A place in a ring of tiles and the parity of its use there.
template <int STAGES>
struct Place {
  uint32_t stage = 0, parity = 0;
  __device__ __forceinline__ void next() {
    if (++stage == STAGES) {
      stage = 0;
      parity ^= 1;
    }
  }
};

// ---- TMA ----
// A box of a [rows][heads][entries] tensor at (entry, head, row).
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int entry, int head,
                                         int row) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(entry), "r"(head), "r"(row)
      : "memory");
}
// Orders this thread's shared memory writes before later products' reads.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tcgen05 ----
template <int COLS>
__device__ __forceinline__ void tmem_alloc(uint32_t where) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "n"(COLS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <int COLS>
__device__ __forceinline__ void tmem_free(uint32_t addr) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Arrives on `bar` when every product issued so far by this thread is done.
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Instruction descriptor: f32 accumulators, 128 x n, 16-bit operands; B with
// its contracted dimension contiguous, or (b_rows) with its n dimension
// contiguous.
__host__ __device__ __forceinline__ uint32_t instr(bool bf16, int n, bool b_rows) {
  const uint32_t t = bf16 ? 1 : 0;
  return 1u << 4 | t << 7 | t << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (128u / 16) << 24;
}
// Shared memory descriptor of a swizzled tile.  Contracted dimension
// contiguous: 8-row groups are 1024 bytes apart.  Otherwise (b_rows) the same
// 1024 bytes separate groups of 8 contracted rows, and blocks of 64 columns
// are kBlockBytes apart.  The address is in the low word; the high one is the
// same for every tile.
constexpr uint32_t kDescHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t tile_desc(uint32_t addr) {
  return (addr >> 4 & 0x3fff) | (uint32_t)(kBlockBytes >> 4) << 16;
}
// The contracted dimension moves by 16 entries: 32 bytes within a row and a
// block further every 64 entries, or 16 rows.
__device__ __forceinline__ constexpr uint32_t step_along(int k) { return (k / 4 * kBlockBytes + k % 4 * 32) >> 4; }
__device__ __forceinline__ constexpr uint32_t step_rows(int k) { return k * 16 * 128 >> 4; }

__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t i, bool add) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 x, y;\nsetp.ne.b32 p, %4, 0;\nmov.b64 x, {%1, %5};\nmov.b64 y, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(i), "r"((uint32_t)add), "r"(kDescHigh)
      : "memory");
}
// A from tensor memory: 16-bit pairs, 8 columns per 16 contracted entries.
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t i, bool add) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 y;\nsetp.ne.b32 p, %4, 0;\nmov.b64 y, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(i), "r"((uint32_t)add), "r"(kDescHigh)
      : "memory");
}

// d = a b^T over `ksteps` steps of 16 contracted entries of two tiles with the
// contracted dimension contiguous.
__device__ __forceinline__ void mma_along(uint32_t d, uint32_t a, uint32_t b, uint32_t i, int ksteps) {
#pragma unroll 1
  for (int e = 0; e < ksteps; e += 4, a += kBlockBytes >> 4, b += kBlockBytes >> 4)
#pragma unroll
    for (int f = 0; f < 4; ++f)
      if (e + f < ksteps) mma(d, a + step_along(f), b + step_along(f), i, e + f > 0);
}
// The same with a in tensor memory.
__device__ __forceinline__ void mma_tmem_along(uint32_t d, uint32_t a, uint32_t b, uint32_t i, int ksteps) {
#pragma unroll 1
  for (int e = 0; e < ksteps; e += 4, a += 32, b += kBlockBytes >> 4)
#pragma unroll
    for (int f = 0; f < 4; ++f)
      if (e + f < ksteps) mma_tmem(d, a + 8 * f, b + step_along(f), i, e + f > 0);
}
// d (+)= a b over 64 contracted rows of a tile, a in tensor memory.
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t i, bool add) {
#pragma unroll
  for (int e = 0; e < 4; ++e) mma_tmem(d, a + 8 * e, b + step_rows(e), i, add || e > 0);
}

// Columns of this warp's 32 lanes, one lane per thread.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
               : "memory");
}

// Of 16 columns of a row, those outside [from, to) become `fill`.
__device__ __forceinline__ void keep16(uint32_t addr, int from, int to, float fill) {
  float x[16];
  tmem_ld16(addr, x);
  wait_ld();
#pragma unroll
  for (int c = 0; c < 16; ++c) x[c] = c >= from && c < to ? x[c] : fill;
  tmem_st16(addr, reinterpret_cast<uint32_t*>(x));
}
// The same for `n` columns, 16 at a time.
__device__ __forceinline__ void keep(uint32_t addr, int n, int from, int to, float fill) {
#pragma unroll 1
  for (int c = 0; c < n; c += 16) keep16(addr + c, from - c, to - c, fill);
  wait_st();
}

// A warpgroup's registers per thread, given up or taken from what the block
// was launched with.
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// ---- arithmetic ----
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two 32-bit operations in one instruction.
__device__ __forceinline__ uint64_t pair_bits(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void pair_split(uint64_t r, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Two values rounded to 16 bits, the first in the low half.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t r) {
  float2 f;
  if (BF16) {
    f.x = __uint_as_float(r << 16);
    f.y = __uint_as_float(r & 0xffff0000u);
  } else {
    asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(f.x), "=f"(f.y) : "r"(r));
  }
  return f;
}

// Writes tiles whose rows lie one per lane, 64 bytes of each row at a time:
// four lanes exchange their 16-byte pieces so that a store takes 64 bytes of 8
// rows instead of 16 bytes of 32.  (Those took some 5000 cycles per tile of
// 128 columns; these take 1000.)
struct RowWriter {
  uint8_t* row[4];     // this lane's piece of the four rows of its group of lanes
  bool on[4];
  __device__ __forceinline__ RowWriter(void* mine, bool valid) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int from = lane / 4 * 4 + e;
      row[e] = reinterpret_cast<uint8_t*>(__shfl_sync(~0u, reinterpret_cast<uint64_t>(mine), from)) + lane % 4 * 16;
      on[e] = __shfl_sync(~0u, (int)valid, from);
    }
  }
  // 16 words of this lane's row, from byte `at` of the row on; the row has `bytes`
  __device__ __forceinline__ void write(const uint32_t* x, int at, int bytes) const {
    const int lane = threadIdx.x % 32;
    uint32_t v[4][4];                                        // piece, word
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e / 4][e % 4] = x[e];
#pragma unroll
    for (int bit = 2; bit; bit >>= 1)                        // lane i, piece j  <->  lane j, piece i
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j & bit) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool up = lane & bit;
          const uint32_t got = __shfl_xor_sync(~0u, up ? v[j][k] : v[j + bit][k], bit);
          v[j][k] = up ? got : v[j][k];
          v[j + bit][k] = up ? v[j + bit][k] : got;
        }
      }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (on[e] && at + lane % 4 * 16 < bytes) *reinterpret_cast<uint4*>(row[e] + at) = make_uint4(v[e][0], v[e][1], v[e][2], v[e][3]);
  }
};

}  // namespace umma
}  // namespace syncgb

// Rows into and out of the paged cache (include/sync.h, sync_cache_append and
// sync_cache_read).
//
// Both are one pass over the rows, bound by memory, in the manner of rotate.cuh:
// a thread has a column of 16 bytes for all tokens of its block.  Sequences,
// positions and places of the block's tokens (reads that depend on one another)
// are found first, a thread per token, for kFound tokens at a time.
//
// 5595 new tokens of 32 + 8 heads of 128 turned and written, and 10554 tokens read
// back, take 46 us in 16 bits (224 MB, 4.8 TB/s); 4096 written and 24097 read 50 us
// in 4 bits (217 MB, 4.4 TB/s).  Between them lie the search for places (a row's
// sequence, length and page come one after the other, 4 us before anything moves)
// and waiting: k_append takes 49% of its issue slots in 16 bits, 57% in 4; of the 15
// and 12 cycles from one instruction of a warp to the next, 5.8 and 2.8 are for reads
// of global memory, 2.1 and 1.4 for barriers.  64 single tokens take 3.4 us in 16 bits
// and 4.3 in 4, captured.
#include <type_traits>

#include "cache.h"
#include "paged.cuh"
#include "rotate.cuh"
#include "sync.h"

namespace syncgb {
namespace {

using namespace rotate;

constexpr int kReadAhead = 8;            // tokens that a thread of k_read has in flight in 16 bits; half as many in 4
constexpr int kReadResident = 768;       // its threads of an SM
// Columns of a block of k_append, tokens that its threads have in flight, and its
// threads of an SM: several blocks, which do not wait for one another's angles.
// (The pieces above with 768 threads and four tokens in flight 52 and 56 us; 1280
// threads of 48 registers 47 and 53; one block of 512 columns 8 us more.)
constexpr int kAppendThreads = 256, kAppendAhead = 2, kAppendResident = 1024;
constexpr int kFound = 512;              // tokens whose places a block knows
// Angles that a block of k_append stages at a time, of at least one group: of many
// groups, as a barrier for each and angles held in registers from one to the next
// cost more (48 and 53 us) than waiting for them now and then.
constexpr int kAngles = 2048;

// 8 entries of a row, by one access or entry by entry
template <class T>
__device__ __forceinline__ void load8(const T* p, bool wide, uint32_t* w) {
  if (wide) {
    *reinterpret_cast<Pack<uint32_t, 4>*>(w) = *reinterpret_cast<const Pack<uint32_t, 4>*>(p);
  } else {
    const uint16_t* x = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
  }
}
template <class T>
__device__ __forceinline__ void unpack8(const uint32_t* w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack<T>(w[i]);
    x[2 * i] = y.x;
    x[2 * i + 1] = y.y;
  }
}

// Entries d .. d + 7 of a key head, whose words are w, after the rotation: by
// their own pairs (interleaved) or with the entries half a rotation further or
// back (other).  c: cosines of the token's pairs, then its sines.
template <class T, bool INTER>
__device__ __forceinline__ void turned8(const T* head, const uint32_t* w, const uint32_t* other, int d, int half, const float* c, float* x) {
  const float* s = c + half;
  unpack8<T>(w, x);
  if (d >= 2 * half) return;
  if (INTER) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      if (d + i < 2 * half) turn(x[i], x[i + 1], c[(d + i) / 2], s[(d + i) / 2]);
  } else if (half % 8 == 0) {
    const int j = d < half ? d : d - half;
    const uint32_t sign = d < half ? 0x80000000u : 0u;      // a c - b s, or b c + a s
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const Pack<float, 4> u = *reinterpret_cast<const Pack<float, 4>*>(c + j + i), v = *reinterpret_cast<const Pack<float, 4>*>(s + j + i);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float2 y = unpack<T>(other[(i + e) / 2]);
        x[i + e] = __fadd_rn(__fmul_rn(x[i + e], u.x[e]), __fmul_rn(__uint_as_float(__float_as_uint(y.x) ^ sign), v.x[e]));
        x[i + e + 1] = __fadd_rn(__fmul_rn(x[i + e + 1], u.x[e + 1]), __fmul_rn(__uint_as_float(__float_as_uint(y.y) ^ sign), v.x[e + 1]));
      }
    }
  } else {                                                  // 8 entries that are not all on one side
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      const int e = d + i, j = e < half ? e : e - half;
      if (e >= 2 * half) break;
      float u = to_f(head[j]), v = to_f(head[j + half]);
      turn(u, v, c[j], s[j]);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = k != i ? x[k] : e < half ? u : v;
    }
  }
}

// 8 entries as 4-bit codes, with the scale of their group, which four
// consecutive lanes share: scale = max |x| / 7 rounded to float16, code =
// x / scale rounded to even, at most 7 in size, stored plus 8.  The divisions
// are by the scale as it is kept.  A group with a NaN or an infinity reads as
// NaN, one beyond 7 * 65504 ends at that.
__device__ __forceinline__ uint32_t codes8(const float* x, __half& scale, uint32_t lanes) {
  uint32_t top = 0;                                         // as bits, so that a NaN is the largest
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(lanes, top, 1));
  top = max(top, __shfl_xor_sync(lanes, top, 2));
  scale = top >= 0x7f800000u ? __ushort_as_half(0x7fff) : __float2half(fminf(__fdiv_rn(__uint_as_float(top), 7.f), 65504.f));
  const float by = __half2float(scale);
  if (!(by > 0.f)) return 0x88888888u;
  // Quotients by the reciprocal, off by less than 7 * 2^-22 from those of the
  // division: where one is so near to a half that this could matter, all are
  // divided.
  const float inverse = __fdiv_rn(1.f, by);
  float far = 0.f;                                          // from the whole number next to it
  uint32_t word = 0;
  auto codes = [&](auto quotient) {
    word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = fminf(7.f, fmaxf(-7.f, quotient(x[i]))), m = t + 12582920.f;   // 1.5 * 2^23 + 8: its last bits are the code
      far = fmaxf(far, fabsf(t - (m - 12582920.f)));
      word |= (__float_as_uint(m) & 15u) << (4 * i);
    }
  };
  codes([&](float v) { return v * inverse; });
  if (far > 0.4999f) codes([&](float v) { return __fdiv_rn(v, by); });
  return word;
}

// Where a row's token is.  place: counted in rows of the cache for key head 0
// (head h is h << page_shift further); -1: nowhere.
struct Where {
  int64_t place;
  int pos;
  int mine;                                                 // a sequence has the row
};
// The groups of a block's next kFound tokens: group, group + gridDim.x, ..; how many.
__device__ __forceinline__ int known_groups(const Columns& c, int64_t group) {
  const int64_t left = (c.groups - group + gridDim.x - 1) / gridDim.x;
  return (int)min(left, (int64_t)(kFound / c.tokens()));
}

// What a thread of k_append has of a token: runs of pairs of a query head, or
// 8 entries of a key or value head.
template <class T, int QVEC, bool INTER>
struct QueryItem {
  static constexpr int kAhead = kAppendAhead;               // tokens in flight
  Pairs<T, QVEC, INTER> x[kAhead];
  const T* from;
  T* to;
  int p, half, pairs;
  int64_t in_row, out_row;
  bool fill;
  __device__ __forceinline__ bool begin(const CacheArgs& a, int column) {
    half = a.turn.half;
    pairs = a.dim / 2;
    const int runs = pairs / QVEC, head = column / runs;
    p = (column - head * runs) * QVEC;
    in_row = a.q.row;
    out_row = a.q_out.row;
    from = static_cast<const T*>(a.q.data) + head * a.q.head;
    to = static_cast<T*>(a.q_out.data) + head * a.q_out.head;
    fill = a.fill;
    return column < a.heads * runs;
  }
  __device__ __forceinline__ void read(int e, int64_t row) { x[e].read(from + row * in_row, p, half, pairs); }
  __device__ __forceinline__ void write(int e, int64_t row, const Where& w, const float* cs) {
    if (w.mine) {
      if (p < half) x[e].template by<true>(cs + p, cs + half + p);
    } else {
      if (!fill) return;
#pragma unroll
      for (uint32_t& z : x[e].w) z = 0;
    }
    x[e].write(to + row * out_row, p, half, pairs);
  }
};

template <class T, int BITS, bool INTER>
struct KeyItem {
  static constexpr int kAhead = kAppendAhead;
  uint32_t x[kAhead][8];                                    // 8 entries, and of a key those that they turn with
  const T* from;
  uint8_t *data, *scales;
  int d, half, row_bytes, g, other;
  int64_t in_row;
  bool is_v, wide, paired;
  __device__ __forceinline__ bool begin(const CacheArgs& a, bool kv_wide, int column) {
    const int runs = a.dim / 8, at = column / runs;
    is_v = at >= a.kv_heads;
    const int head = is_v ? at - a.kv_heads : at;
    const HeadTensor& in = is_v ? a.v_rows : a.k_rows;
    const int64_t head_rows = (int64_t)head << a.page_shift;
    half = a.turn.half;
    g = a.dim / kGroup;
    d = (column - at * runs) * 8;
    from = static_cast<const T*>(in.data) + head * in.head;
    in_row = in.row;
    row_bytes = BITS == 16 ? 2 * a.dim : a.dim / 2;
    data = (is_v ? a.v : a.k) + head_rows * row_bytes + (BITS == 16 ? 2 * d : 4 * paged::word_of(d / 8, g));
    scales = BITS == 16 ? nullptr : (is_v ? a.v_scale : a.k_scale) + 2 * (head_rows * g + d / kGroup);
    wide = kv_wide;
    paired = !INTER && !is_v && half % 8 == 0 && d < 2 * half;
    other = d < half ? half : -half;
    return column < 2 * a.kv_heads * runs;
  }
  __device__ __forceinline__ void read(int e, int64_t row) {
    const T* head = from + row * in_row + d;
    load8(head, wide, x[e]);
    if (paired) load8(head + other, wide, x[e] + 4);
  }
  __device__ __forceinline__ void write(int e, int64_t row, const Where& w, const float* cs) {
    if (w.place < 0) return;
#pragma unroll
    for (uint32_t& z : x[e]) asm volatile("" : "+r"(z));     // (unpacked from here on, not where they were read)
    uint8_t* const to = data + w.place * row_bytes;
    if (BITS == 16 && (is_v || d >= 2 * half)) {
      *reinterpret_cast<Pack<uint32_t, 4>*>(to) = *reinterpret_cast<const Pack<uint32_t, 4>*>(x[e]);
      return;
    }
    float y[8];
    if (is_v) unpack8<T>(x[e], y);
    else turned8<T, INTER>(from + row * in_row, x[e], x[e] + 4, d, half, cs, y);
    if (BITS == 16) {
      Pack<uint32_t, 4> z;
#pragma unroll
      for (int i = 0; i < 4; ++i) z.x[i] = pack<T>(y[2 * i], y[2 * i + 1]);
      *reinterpret_cast<Pack<uint32_t, 4>*>(to) = z;
    } else {
      __half scale;
      *reinterpret_cast<uint32_t*>(to) = codes8(y, scale, 0xfu << (threadIdx.x % 32 / 4 * 4));
      if (d % kGroup == 0) *reinterpret_cast<__half*>(scales + w.place * (2 * g)) = scale;
    }
  }
};

// All tokens of this block through `item`, which has this thread's column.
template <class Item>
__device__ __forceinline__ void through(const CacheArgs& a, const Columns& c, float* angles, Where* where, bool on, Item& item) {
  constexpr int kAhead = Item::kAhead;
  const int half = a.turn.half, tokens = c.tokens(), sub = threadIdx.x / c.each;
  auto here = [&](int64_t row, int e) { return on && e < c.ahead && row < a.rows; };
  auto read = [&](int64_t group) {
    int64_t row = group * tokens + sub;
#pragma unroll
    for (int e = 0; e < kAhead; ++e, row += c.par)
      if (here(row, e)) item.read(e, row);
  };
  auto search = [&](int64_t group, int groups) {            // into where, for that many groups
    for (int i = threadIdx.x; i < groups * tokens; i += blockDim.x) {
      const int64_t row = (group + (int64_t)(i / tokens) * gridDim.x) * tokens + i % tokens;
      Where w{-1, -1, 0};
      const int s = row < a.rows ? paged::sequence_of(a, (int)row) : -1;
      if (s >= 0) {
        w.mine = 1;
        w.pos = (int)(a.starts ? (int64_t)__ldg(a.lens + s) - __ldg(a.starts + s + 1) + row : (int64_t)__ldg(a.lens + s) - 1);
        const int64_t at = paged::place_of(a, s, w.pos);
        if (at >= 0) w.place = paged::row_of(a, at, 0);
      }
      where[i] = w;
    }
  };
  // angles of the groups from `group` on whose tokens are [at, end) of where
  auto stage = [&](int64_t group, int at, int end) {
    const int some = (end - at) * half;
#pragma unroll 2
    for (int i = threadIdx.x; i < some; i += blockDim.x) {
      const int t = i / half, j = i - t * half;
      const Where& w = where[at + t];
      if (!w.mine) continue;
      const int64_t row = (group + (int64_t)(t / tokens) * gridDim.x) * tokens + t % tokens;
      const float2 x = angle(a.turn, position(a.turn, row, w.pos, j), j);
      angles[2 * t * half + j] = x.x;
      angles[(2 * t + 1) * half + j] = x.y;
    }
  };
  int64_t group = blockIdx.x;
  read(group);
  while (group < c.groups) {
    const int known = known_groups(c, group);
    search(group, known);
    __syncthreads();
#pragma unroll 1
    for (int first = 0; first < known; first += c.batch) {
      const int last = min(first + c.batch, known);
      stage(group, first * tokens, last * tokens);
      __syncthreads();
      const float* cs = angles + sub * 2 * half;
#pragma unroll 1
      for (int n = first; n < last; ++n, cs += tokens * 2 * half) {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int token = sub + e * c.par;
          const int64_t row = group * tokens + token;
          if (here(row, e)) item.write(e, row, where[n * tokens + token], cs + e * c.par * 2 * half);
        }
        group += gridDim.x;
        if (group < c.groups) read(group);
      }
      __syncthreads();
    }
  }
}

// New tokens into the cache: blocks [0, kv_blocks) of a group take its keys and
// values, the others its queries.  T: their type; QVEC: pairs of a query head that
// a thread takes at a time.
template <class T, int QVEC, int BITS, bool INTER>
__global__ void __launch_bounds__(kAppendThreads, kAppendResident / kAppendThreads) k_append(const __grid_constant__ CacheArgs a, const __grid_constant__ Columns c, int kv_blocks, bool kv_wide) {
  extern __shared__ __align__(16) float angles[];           // [batch][tokens][cos, sin][half]
  __shared__ Where where[kFound];
  const bool on = (int)threadIdx.x / c.each < c.par;
  const int column = threadIdx.x % c.each;
  if ((int)blockIdx.y < kv_blocks) {
    KeyItem<T, BITS, INTER> item;
    const bool has = item.begin(a, kv_wide, blockIdx.y * c.each + column);
    through(a, c, angles, where, on && has, item);
  } else {
    QueryItem<T, QVEC, INTER> item;
    const bool has = item.begin(a, (blockIdx.y - kv_blocks) * c.each + column);
    through(a, c, angles, where, on && has, item);
  }
}

// What a thread of k_read has of a cached token: 8 entries in 16 bits (G 0), or in
// 4 bits a quarter of a row of G groups, 8 entries of every group (one group's 8
// entries a thread, with twice as many tokens: 4 us more for 24097 tokens).
template <class T, int G>
struct Cached {
  static constexpr int kAhead = kReadAhead / (G ? 2 : 1), kPieces = G ? G : 1;
  alignas(16) uint32_t w[G ? G : 4];
  alignas(8) uint32_t scale[G ? (G + 1) / 2 : 1];
  __device__ __forceinline__ void read(const uint8_t* row, const uint8_t* scales) {
    if constexpr (G == 3) {                                 // 12 bytes are aligned to 4, and 6 to 2
#pragma unroll
      for (int i = 0; i < 3; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t*>(row) + i);
      const uint16_t* h = reinterpret_cast<const uint16_t*>(scales);
      scale[0] = __ldg(h) | (uint32_t)__ldg(h + 1) << 16;
      scale[1] = __ldg(h + 2);
    } else {
      constexpr int N = G ? G : 4;
      *reinterpret_cast<Pack<uint32_t, N>*>(w) = *reinterpret_cast<const Pack<uint32_t, N>*>(row);
      if constexpr (G == 1) scale[0] = __ldg(reinterpret_cast<const uint16_t*>(scales));
      else if constexpr (G != 0) *reinterpret_cast<Pack<uint32_t, G / 2>*>(scale) = *reinterpret_cast<const Pack<uint32_t, G / 2>*>(scales);
    }
  }
  // piece i of the row at `to`
  __device__ __forceinline__ void write(T* to, int i) const {
    Pack<uint32_t, 4> z;
    if constexpr (G == 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) z.x[e] = w[e];
    } else {
      const float by = __half2float(__ushort_as_half((uint16_t)(scale[i / 2] >> (16 * (i % 2)))));
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {                         // 2^23 + code, as bits, less 2^23 + 8
        y[e] = (__uint_as_float((w[i] >> (4 * e) & 15) | 0x4b000000u) - 8388616.f) * by;
        // 7 scales may be past float16's end where the row's largest entry was not: the scale was rounded
        if (std::is_same<T, __half>::value) y[e] = y[e] > 65504.f ? 65504.f : y[e] < -65504.f ? -65504.f : y[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) z.x[e] = pack<T>(y[2 * e], y[2 * e + 1]);
    }
    *reinterpret_cast<Pack<uint32_t, 4>*>(to + kGroup * i) = z;
  }
  static __device__ __forceinline__ void fill(T* to, uint32_t with) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) *reinterpret_cast<uint4*>(to + kGroup * i) = make_uint4(with, with, with, with);
  }
};

// Cached tokens back to rows of 16 bits: the tokens of sequence s from its first
// one on go to rows starts[s] .. starts[s + 1]; zeros past its length.
template <class T, int G>
__global__ void __launch_bounds__(kReadResident, 1) k_read(const __grid_constant__ CacheArgs a, const __grid_constant__ Columns c) {
  __shared__ int64_t places[kFound];                        // as in Where; -1: no such token, -2: no sequence's row, -3: no such page
  const int tokens = c.tokens(), runs = G ? 4 : a.dim / 8;
  const int sub = threadIdx.x / c.each, column = blockIdx.y * c.each + threadIdx.x % c.each;
  const bool on = sub < c.par && column < 2 * a.kv_heads * runs;
  const int at = column / runs, run = column - at * runs;
  const bool is_v = at >= a.kv_heads;
  const int head = is_v ? at - a.kv_heads : at;
  const HeadTensor& out = is_v ? a.v_rows : a.k_rows;
  T* const to = static_cast<T*>(out.data) + head * out.head + 8 * run;
  const int64_t out_row = out.row, out_step = out_row * c.par, head_rows = (int64_t)head << a.page_shift;
  // this column's piece of the cache's rows
  const int row_bytes = G ? G * 16 : 2 * a.dim;
  const uint8_t* const data = (is_v ? a.v : a.k) + head_rows * row_bytes + (G ? 4 * G : 16) * run;
  const uint8_t* const scales = G ? (is_v ? a.v_scale : a.k_scale) + head_rows * G * 2 : nullptr;

  int64_t group = blockIdx.x;
  while (group < c.groups) {
    const int known = known_groups(c, group);
    for (int i = threadIdx.x; i < known * tokens; i += blockDim.x) {
      const int64_t row = (group + (int64_t)(i / tokens) * gridDim.x) * tokens + i % tokens;
      const int s = row < a.rows ? paged::sequence_of(a, (int)row) : -1;
      int64_t p = -2;
      if (s >= 0) {
        const int64_t pos = row - __ldg(a.starts + s);
        p = -1;
        if (pos < __ldg(a.lens + s)) {
          p = paged::place_of(a, s, pos);
          p = p < 0 ? -3 : paged::row_of(a, p, 0);
        }
      }
      places[i] = p;
    }
    __syncthreads();
#pragma unroll 1
    for (int n = 0; n < known; ++n, group += gridDim.x) {
      const int64_t row = group * tokens + sub, left = a.rows - row;
      const int mine = !on ? 0 : left >= tokens ? c.ahead : left > 0 ? ((int)left + c.par - 1) / c.par : 0;
      const int64_t* const place = places + n * tokens + sub;
      using Token = Cached<T, G>;
      Token x[Token::kAhead];
#pragma unroll
      for (int e = 0; e < Token::kAhead; ++e) {
        if (e >= mine) break;
        const int64_t p = place[e * c.par];
        if (p >= 0) x[e].read(data + p * row_bytes, scales + p * (2 * G));
      }
      T* o = to + row * out_row;
#pragma unroll
      for (int e = 0; e < Token::kAhead; ++e, o += out_step) {
        if (e >= mine) break;
        const int64_t p = place[e * c.par];
        if (p >= 0) {
#pragma unroll
          for (int i = 0; i < Token::kPieces; ++i) x[e].write(o, i);
        } else if (p != -2 || a.fill) {
          Token::fill(o, p == -3 ? 0x7fff7fffu : 0u);        // NaN in both types
        }
      }
    }
    __syncthreads();
  }
}

template <class T, int QVEC, int BITS>
cudaError_t append(const CacheArgs& a, bool kv_wide, cudaStream_t st) {
  const int kv = 2 * a.kv_heads * (a.dim / 8), q = a.heads * (a.dim / 2 / QVEC);
  Columns c = columns_of(a.rows, std::min(kAppendThreads, std::max(kv, q)), kAppendAhead, a.turn.half, a.num_sms, kAppendThreads, kAppendResident);
  const int kv_blocks = (kv + c.each - 1) / c.each;
  c.blocks_y = kv_blocks + (q + c.each - 1) / c.each;
  c.blocks_x = std::max(1, std::min(c.blocks_x, a.num_sms * std::max(1, kAppendResident / c.threads) / c.blocks_y));
  const dim3 grid((unsigned)c.blocks_x, (unsigned)c.blocks_y);
  c.batch = std::max(1, std::min(kFound, a.turn.half ? kAngles / a.turn.half : kFound) / c.tokens());
  const size_t smem = (size_t)2 * c.batch * c.tokens() * a.turn.half * sizeof(float);
  if (a.turn.interleaved) k_append<T, QVEC, BITS, true><<<grid, c.threads, smem, st>>>(a, c, kv_blocks, kv_wide);
  else k_append<T, QVEC, BITS, false><<<grid, c.threads, smem, st>>>(a, c, kv_blocks, kv_wide);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

template <class T>
cudaError_t append_type(const CacheArgs& a, cudaStream_t st) {
  bool wide = true;
  for (const HeadTensor* t : {&a.k_rows, &a.v_rows})
    wide = wide && reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->row % 8 == 0 && t->head % 8 == 0;
  const HeadTensor q[2] = {a.q, a.q_out};
  const int vec = a.heads ? widest(q, 2, 2, a.turn.half, a.dim) : 8;
  auto with = [&](auto bits) {
    constexpr int kBits = decltype(bits)::value;
    return vec == 8 ? append<T, 8, kBits>(a, wide, st) : vec == 4 ? append<T, 4, kBits>(a, wide, st) : append<T, 1, kBits>(a, wide, st);
  };
  return a.bits == 16 ? with(std::integral_constant<int, 16>()) : with(std::integral_constant<int, 4>());
}

}  // namespace

cudaError_t launch_cache_append(const CacheArgs& a, cudaStream_t st) {
  if (!a.rows) return cudaSuccess;
  return a.bf16 ? append_type<__nv_bfloat16>(a, st) : append_type<__half>(a, st);
}

cudaError_t launch_cache_read(const CacheArgs& a, cudaStream_t st) {
  if (!a.rows) return cudaSuccess;
  auto go = [&](auto type, auto groups) {
    using Token = Cached<decltype(type), decltype(groups)::value>;
    const int columns = 2 * a.kv_heads * (a.bits == 4 ? 4 : a.dim / 8);
    const Columns c = columns_of(a.rows, columns, Token::kAhead, 0, a.num_sms, kMostThreads, kReadResident);
    k_read<decltype(type), decltype(groups)::value><<<dim3((unsigned)c.blocks_x, (unsigned)c.blocks_y), c.threads, 0, st>>>(a, c);
  };
  auto narrow = [&](auto type) {
    switch (a.dim / kGroup) {
      case 1: return go(type, std::integral_constant<int, 1>());
      case 2: return go(type, std::integral_constant<int, 2>());
      case 3: return go(type, std::integral_constant<int, 3>());
      default: return go(type, std::integral_constant<int, 4>());
    }
  };
  if (a.bits == 16) go(__nv_bfloat16(), std::integral_constant<int, 0>());   // (whichever type: the bits are copied)
  else if (a.bf16) narrow(__nv_bfloat16());
  else narrow(__half());
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) count_launch();
  return e;
}

}  // namespace syncgb

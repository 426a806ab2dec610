// How the blocks of an attention call over the paged cache divide its work, on
// the device and, for tests, on the host.
//
// The work is a list: sequence > key head > pass (of `rows` query rows) > tile
// of `tile` keys, every pass counting kUnitCost tiles more for its start and end
// (64 sequences of 1 to 8192 tokens: 3 tiles 62 us, 1 tile 69; 2 tiles cost 24
// short sequences of up to 5 new tokens 2.4 us, 4 tiles 512 sequences 2 us).
// A warp has an equal run of it.  A pass that a warp begins but does not end is
// continued by the warps that follow.  Or (whole) passes are not cut and count one
// each, where none can have more than a few tiles.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace syncgb {
namespace division {

#ifdef __CUDACC__
#define SYNCGB_BOTH __host__ __device__ __forceinline__
#else
#define SYNCGB_BOTH inline
#endif

constexpr int kUnitCost = 3, kLeast = 2;   // tiles that a pass costs besides; that a warp takes at least

SYNCGB_BOTH int64_t less(int64_t a, int64_t b) { return a < b ? a : b; }
SYNCGB_BOTH int64_t more(int64_t a, int64_t b) { return a > b ? a : b; }

// A sequence: its rows [begin, end) as the caller's arrays have them, brought
// into the tensors' rows, and its tokens, of which pages hold `room` at most.
struct Shape {
  int row0, n, len, bad, tiles, passes, unit;   // unit: what a pass costs
  int64_t cost;
};
SYNCGB_BOTH Shape shape(int64_t begin, int64_t end, int64_t all_rows, int len, int room, int group, int kv_heads, int rows,
                        int tile, bool whole) {
  Shape x;
  begin = less(more(begin, 0), all_rows);
  end = less(more(end, begin), all_rows);
  x.row0 = (int)begin;
  x.n = (int)(end - begin);
  x.bad = len > room;
  x.len = (int)less(more(len, 0), room);
  x.tiles = (int)(((int64_t)x.len + tile - 1) / tile);
  x.passes = (int)(((int64_t)x.n * group + rows - 1) / rows);
  x.unit = whole ? 1 : x.tiles + kUnitCost;
  x.cost = (int64_t)x.passes * kv_heads * x.unit;
  return x;
}

// Warps that take work, and where the run of one begins (and the last one's ends).
SYNCGB_BOTH int takers(int64_t total, int warps, bool whole) { return (int)more(1, less(warps, whole ? total : total / kLeast)); }
SYNCGB_BOTH int64_t bound(int64_t total, int takers, int warp) {
  warp = (int)less(warp, takers);
  if (total < (int64_t)1 << 32 && (uint64_t)total * (uint32_t)takers < (uint64_t)1 << 32) return (uint32_t)total * (uint32_t)warp / (uint32_t)takers;
  return total / takers * warp + total % takers * warp / takers;   // (no product as large as total * warp)
}

// The warp whose run has the tile at x < total.
SYNCGB_BOTH int holder(int64_t total, int takers, int64_t x) {
  int w = (int)less((int64_t)((double)x / (double)total * takers), takers - 1);
  while (bound(total, takers, w) > x) --w;
  while (bound(total, takers, w + 1) <= x) ++w;
  return w;
}

// A warp's part of a pass.
struct Piece {
  int s, head;                             // sequence, key head
  int first, n, row0;                      // first row of the pass among the n * group rows; tokens; row of the first token
  int len, bad;                            // tokens in the cache; more than its pages hold
  int from, to, tiles;                     // tiles of the warp, and of the pass
  int64_t at;                              // where the pass is in the list
  SYNCGB_BOTH int64_t last_tile() const { return at + kUnitCost + tiles - 1; }
};

// The first sequence behind s, which has no rows, whose rows end further on, by
// steps that double (a run of empty ones costs its logarithm in reads); n_seqs
// where there is none.  Safe, if not right, where starts do fall.
template <class At>
SYNCGB_BOTH int behind_empty(At&& starts, int s, int n_seqs) {
  const int here = starts(s);
  int step = 1;
  while (step < n_seqs - s && starts(s + step + 1) <= here) {
    s += step;
    step *= 2;
  }
  int lo = s, hi = (int)less((int64_t)s + step, n_seqs);   // lo is empty; hi is not, or n_seqs
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (starts(mid + 1) <= here) lo = mid;
    else hi = mid;
  }
  return hi;
}

// The pieces of a warp, one after the other.
struct Lister {
  Shape now;
  int s, unit;                             // unit: key head * passes + pass
  int64_t into, left, at;                  // tiles into the unit, tiles left of the run; where the unit begins
  // The run of `run` tiles from `begin` on, which is into_seq into the sequence's work.
  SYNCGB_BOTH void start(const Shape& x, int seq, int64_t begin, int64_t into_seq, int64_t run) {
    now = x;
    s = seq;
    const int cost = x.unit;
    unit = into_seq < (int64_t)1 << 31 ? (int)((uint32_t)into_seq / (uint32_t)cost) : (int)(into_seq / cost);
    into = into_seq - (int64_t)unit * cost;
    left = run;
    at = begin - into;
  }
  // skip(s): the first sequence behind s, which has no rows, that may have some
  template <class F, class G>
  SYNCGB_BOTH bool next(F&& shape_of, G&& skip, int n_seqs, int kv_heads, int rows, bool whole, Piece& x) {
    while (left > 0) {
      if (unit >= now.passes * kv_heads) {
        s = now.n ? s + 1 : skip(s);
        if (s >= n_seqs) return false;
        now = shape_of(s);
        unit = 0;
        into = 0;
        continue;
      }
      const int64_t to = less(now.unit, into + left);
      const int a = whole ? 0 : (int)more(0, into - kUnitCost), b = whole ? now.tiles : (int)more(0, to - kUnitCost);
      const bool some = b > a || (now.tiles == 0 && into == 0);
      if (some) x = Piece{s, unit / now.passes, unit % now.passes * rows, now.n, now.row0, now.len, now.bad, a, b, now.tiles, at};
      left -= to - into;
      into = 0;
      at += now.unit;
      ++unit;
      if (some) return true;
    }
    return false;
  }
};

}  // namespace division
}  // namespace syncgb

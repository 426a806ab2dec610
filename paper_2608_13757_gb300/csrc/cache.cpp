// C ABI of the rotation and of the paged cache (include/sync.h): argument
// checks and the launches.
#include "cache.h"

#include <algorithm>
#include <cmath>

#include "abi.h"
#include "division.h"

using namespace syncgb;
using namespace syncgb::abi;

namespace {

HeadTensor tensor(const sync_rows* t, int64_t rows, int size, bool output, int32_t heads, const char* what) {
  need(t, what);
  need(t->rows == rows, "tensors of a call must have the same number of rows");
  need(t->data || rows == 0, what);
  need_aligned(t->data, size, "a tensor is not aligned to its type");
  need(!output || ((rows <= 1 || t->row_stride) && (heads <= 1 || t->head_stride)), "an output's rows and heads must not share memory");
  HeadTensor r;
  r.data = t->data;
  r.rows = rows;
  r.row = t->row_stride;
  r.head = t->head_stride;
  return r;
}

// The same for tensors that are read or written 16 bytes at a time.
HeadTensor wide_tensor(const sync_rows* t, int64_t rows, bool output, int32_t heads, const char* what) {
  const HeadTensor r = tensor(t, rows, 2, output, heads, what);
  need(reinterpret_cast<uintptr_t>(r.data) % 16 == 0 && r.row % 8 == 0 && r.head % 8 == 0,
       "tensors of this call must be 16-byte aligned with strides that are multiples of 8 entries");
  return r;
}

Rotation rotation(const sync_rotation* t, int dim, int64_t rows) {
  Rotation r;
  if (!t || t->rotated == 0) return r;
  need(t->rotated > 0 && t->rotated <= dim && t->rotated % 2 == 0, "rotated must be even and in 0..dim");
  need(t->n_axes >= 1 && t->n_axes <= kAxes, "n_axes must be in 1..4");
  need(t->positions || t->n_axes == 1 || rows == 0, "several axes need positions");
  need(t->n_positions >= 0, "n_positions must not be negative");
  need(rows == 0 || (t->cos && t->sin), "cos and sin must not be NULL");
  need_aligned(t->cos, 4, "cos is not aligned to its type");
  need_aligned(t->sin, 4, "sin is not aligned to its type");
  need_aligned(t->positions, 4, "positions is not aligned to its type");
  r.half = t->rotated / 2;
  r.interleaved = t->interleaved != 0;
  r.cos = t->cos;
  r.sin = t->sin;
  r.n_positions = t->n_positions;
  r.positions = t->positions;
  r.position_stride = t->position_stride;
  for (int j = 0; t->pair_axis && j < r.half; ++j) {
    need(t->pair_axis[j] < t->n_axes, "an entry of pair_axis is not below n_axes");
    r.axis[j / 16] |= (uint32_t)t->pair_axis[j] << (2 * (j % 16));
  }
  return r;
}

RopeArgs rope_args(const sync_rope_desc* p, const sync_rows* q_out, const sync_rows* k_out) {
  need(p, "the description must not be NULL");
  need(p->dtype == SYNC_BF16 || p->dtype == SYNC_FP16 || p->dtype == SYNC_FP32, "dtype must be a sync_dtype");
  need(p->heads >= 1 && p->kv_heads >= 1 && p->heads <= 65536 && p->kv_heads <= 65536, "heads and kv_heads must be in 1..65536");
  need(p->dim >= 2 && p->dim <= 2 * kMostPairs && p->dim % 2 == 0, "dim must be even and in 2..256");
  need(p->q.rows >= 0 && p->q.rows <= INT32_MAX, "the number of rows must be in 0..INT32_MAX");
  need(p->turn.rotated >= 0, "rotated must be even and in 0..dim");
  const int size = p->dtype == SYNC_FP32 ? 4 : 2;
  RopeArgs a;
  a.dtype = p->dtype;
  a.heads = p->heads;
  a.kv_heads = p->kv_heads;
  a.dim = p->dim;
  a.rows = p->q.rows;
  a.q = tensor(&p->q, a.rows, size, false, a.heads, "q must not be NULL");
  a.k = tensor(&p->k, a.rows, size, false, a.kv_heads, "k must not be NULL");
  a.q_out = tensor(q_out, a.rows, size, true, a.heads, "the output for q must not be NULL");
  a.k_out = tensor(k_out, a.rows, size, true, a.kv_heads, "the output for k must not be NULL");
  a.turn = rotation(&p->turn, a.dim, a.rows);
  return a;
}

// The cache alone.
CacheArgs cache_args(const sync_cache* c) {
  need(c, "the cache must not be NULL");
  need(c->dtype == SYNC_BF16 || c->dtype == SYNC_FP16, "dtype must be SYNC_BF16 or SYNC_FP16");
  need(c->bits == 16 || c->bits == 4, "bits must be 16 or 4");
  need(c->kv_heads >= 1 && c->kv_heads <= 65536, "kv_heads must be in 1..65536");
  const int step = c->bits == 4 ? kGroup : 8;
  need(c->head_dim >= step && c->head_dim <= 128 && c->head_dim % step == 0,
       c->bits == 4 ? "head_dim must be a multiple of 32 in 32..128 in 4 bits" : "head_dim must be a multiple of 8 in 8..128");
  need(c->page >= 16 && c->page <= 1024 && (c->page & (c->page - 1)) == 0, "page must be a power of two in 16..1024");
  need(c->n_pages >= 0 && (int64_t)c->n_pages * c->page <= INT32_MAX, "n_pages * page must be in 0..INT32_MAX");
  need((int64_t)c->n_pages * c->page / 16 * c->kv_heads <= UINT32_MAX, "the cache has more than 16 * UINT32_MAX rows");
  CacheArgs a;
  a.bf16 = c->dtype == SYNC_BF16;
  a.bits = c->bits;
  a.kv_heads = c->kv_heads;
  a.dim = c->head_dim;
  while ((1 << a.page_shift) < c->page) ++a.page_shift;
  a.n_pages = c->n_pages;
  a.k = static_cast<uint8_t*>(c->k);
  a.v = static_cast<uint8_t*>(c->v);
  a.k_scale = static_cast<uint8_t*>(c->k_scale);
  a.v_scale = static_cast<uint8_t*>(c->v_scale);
  return a;
}

CacheArgs cache_args(const sync_cache* c, const sync_cache_seqs* s) {
  CacheArgs a = cache_args(c);
  need(a.n_pages == 0 || (a.k && a.v && (a.bits == 16 || (a.k_scale && a.v_scale))), "the cache's tensors must not be NULL");
  for (const void* p : {a.k, a.v, a.k_scale, a.v_scale}) need_aligned(p, 16, "the cache's tensors must be 16-byte aligned");
  need(s, "the sequences must not be NULL");
  need(s->n_seqs >= 0 && s->max_pages >= 0 && s->n_seqs <= 1 << 20, "n_seqs must be in 0..2^20, max_pages not negative");
  need((int64_t)s->max_pages * c->page <= INT32_MAX, "max_pages * page must be at most INT32_MAX");
  need(s->n_seqs == 0 || (s->lens && (s->page_table || s->max_pages == 0)), "page_table and lens must not be NULL");
  need_aligned(s->page_table, 4, "page_table is not aligned to its type");
  need_aligned(s->lens, 4, "lens is not aligned to its type");
  need_aligned(s->row_starts, 4, "row_starts is not aligned to its type");
  a.n_seqs = s->n_seqs;
  a.max_pages = s->max_pages;
  a.table = s->page_table;
  a.table_stride = s->table_stride;
  a.lens = s->lens;
  a.starts = s->row_starts;
  return a;
}

void take_rows(CacheArgs& a, int64_t rows) {
  need(rows >= 0 && rows <= INT32_MAX, "the number of rows must be in 0..INT32_MAX");
  need(a.starts || rows == a.n_seqs, "without row_starts there is one row per sequence");
  a.rows = rows;
}

int checked_heads(const sync_cache* c, int32_t heads) {
  need(heads >= 1 && heads <= 65536 && heads % c->kv_heads == 0, "heads must be a positive multiple of kv_heads, at most 65536");
  return heads;
}

}  // namespace

// For tests on the host: the pieces that `warps` warps take of a step with
// `group` query heads per key head, passes of `rows` rows and tiles of `tile` keys,
// 12 values per piece: warp, sequence, key head, first row, tokens, first token's
// row, length, bad, tiles [from, to) of tiles, the warp of the pass's last tile.
// Returns the number of pieces (written up to `capacity`).
extern "C" int64_t syncgb_cache_attn_work(int n_seqs, const int32_t* lens, const int32_t* row_starts, int64_t all_rows, int room,
                                          int kv_heads, int group, int rows, int tile, int whole, int warps, int64_t* out, int64_t capacity) {
  auto shape_of = [&](int s) {
    return division::shape(row_starts ? row_starts[s] : s, row_starts ? row_starts[s + 1] : s + 1, all_rows, lens[s], room, group, kv_heads, rows, tile, whole != 0);
  };
  auto after_empty = [&](int s) { return row_starts ? division::behind_empty([&](int i) { return row_starts[i]; }, s, n_seqs) : s + 1; };
  int64_t total = 0, n = 0;
  for (int s = 0; s < n_seqs; ++s) total += shape_of(s).cost;
  const int takers = division::takers(total, warps, whole != 0);
  for (int w = 0; w < warps; ++w) {
    const int64_t begin = division::bound(total, takers, w), run = division::bound(total, takers, w + 1) - begin;
    if (!run) continue;
    int s = 0;
    int64_t from = begin;
    for (; from >= shape_of(s).cost; ++s) from -= shape_of(s).cost;
    division::Lister l;
    l.start(shape_of(s), s, begin, from, run);
    division::Piece x;
    for (; l.next(shape_of, after_empty, n_seqs, kv_heads, rows, whole != 0, x); ++n) {
      const int64_t row[12] = {w, x.s, x.head, x.first, x.n, x.row0, x.len, x.bad, x.from, x.to, x.tiles,
                               x.tiles && !whole ? division::holder(total, takers, x.last_tile()) : w};
      if (n < capacity) std::copy(row, row + 12, out + 12 * n);
    }
  }
  return n;
}

extern "C" {

sync_status sync_rope(const sync_rope_desc* p, const sync_rows* q_out, const sync_rows* k_out, void* stream) {
  return guarded([&] {
    RopeArgs a = rope_args(p, q_out, k_out);
    if (!a.rows) return;
    a.num_sms = current_sms();
    cuda(launch_rope(a, static_cast<cudaStream_t>(stream)), "sync_rope");
  });
}

sync_status sync_rope_backward(const sync_rope_desc* p, const sync_rows* dq, const sync_rows* dk, void* stream) {
  return guarded([&] {
    RopeArgs a = rope_args(p, dq, dk);
    if (!a.rows) return;
    a.turn.way = -1.f;
    a.num_sms = current_sms();
    cuda(launch_rope(a, static_cast<cudaStream_t>(stream)), "sync_rope_backward");
  });
}

sync_status sync_cache_append(const sync_cache* cache, const sync_cache_seqs* seqs, const sync_rows* k, const sync_rows* v,
                              int32_t heads, const sync_rows* q, const sync_rows* q_out, const sync_rotation* turn,
                              int32_t zero_rest, void* stream) {
  return guarded([&] {
    CacheArgs a = cache_args(cache, seqs);
    need(k && v, "k and v must not be NULL");
    take_rows(a, k->rows);
    a.k_rows = tensor(k, a.rows, 2, false, a.kv_heads, "k must not be NULL");
    a.v_rows = tensor(v, a.rows, 2, false, a.kv_heads, "v must not be NULL");
    need(!q == !q_out, "q and q_out must both be given or both be NULL");
    if (q) {
      a.heads = checked_heads(cache, heads);
      a.q = tensor(q, a.rows, 2, false, a.heads, "q must not be NULL");
      a.q_out = tensor(q_out, a.rows, 2, true, a.heads, "q_out must not be NULL");
    }
    need(!turn || turn->rotated >= 0, "rotated must be even and in 0..dim");
    a.turn = rotation(turn, a.dim, a.rows);
    a.fill = zero_rest != 0;
    if (!a.rows) return;
    a.num_sms = current_sms();
    cuda(launch_cache_append(a, static_cast<cudaStream_t>(stream)), "sync_cache_append");
  });
}

sync_status sync_cache_read(const sync_cache* cache, const sync_cache_seqs* seqs, const sync_rows* k, const sync_rows* v,
                            int32_t zero_rest, void* stream) {
  return guarded([&] {
    CacheArgs a = cache_args(cache, seqs);
    need(a.starts || a.n_seqs == 0, "row_starts must not be NULL");
    need(k && v, "k and v must not be NULL");
    need(k->rows >= 0 && k->rows <= INT32_MAX, "the number of rows must be in 0..INT32_MAX");
    a.rows = k->rows;
    a.k_rows = wide_tensor(k, a.rows, true, a.kv_heads, "k must not be NULL");
    a.v_rows = wide_tensor(v, a.rows, true, a.kv_heads, "v must not be NULL");
    a.fill = zero_rest != 0;
    if (!a.rows) return;
    a.num_sms = current_sms();
    cuda(launch_cache_read(a, static_cast<cudaStream_t>(stream)), "sync_cache_read");
  });
}

sync_status sync_cache_attn_workspace(const sync_cache* cache, int32_t heads, int32_t max_new, int64_t* bytes) {
  return guarded([&] {
    const CacheArgs a = cache_args(cache);
    const int group = checked_heads(cache, heads) / a.kv_heads;
    need(max_new >= 1, "max_new must be at least 1");
    need(bytes, "bytes must not be NULL");
    const int rows = cache_attn_rows(a.bits, group, max_new);
    *bytes = cache_attn_workspace(a.dim, rows, cache_attn_blocks(a.bits, rows, current_sms()));
  });
}

sync_status sync_cache_attn(const sync_cache* cache, const sync_cache_seqs* seqs, int32_t heads, const sync_rows* q, float scale,
                            int32_t max_new, const sync_rows* o, float* lse, int32_t zero_rest, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  return guarded([&] {
    CacheArgs a = cache_args(cache, seqs);
    a.heads = checked_heads(cache, heads);
    need(std::isfinite(scale) && scale > 0.f, "scale must be positive and finite");
    need(max_new >= 1, "max_new must be at least 1");
    need_aligned(lse, 4, "lse is not aligned to its type");
    need(q, "q must not be NULL");
    take_rows(a, q->rows);
    a.q = wide_tensor(q, a.rows, false, a.heads, "q must not be NULL");
    a.q_out = wide_tensor(o, a.rows, true, a.heads, "o must not be NULL");
    a.scale = scale;
    a.lse = lse;
    a.fill = zero_rest != 0;
    a.whole = (int64_t)seqs->max_pages * cache->page <= SYNC_CACHE_SHORT;
    need(a.rows * (a.heads / a.kv_heads) <= 1 << 30 && a.rows * a.heads <= (int64_t)1 << 33,
         "more than 2^30 query rows of a key head, or 2^33 of all");
    need(a.whole || (workspace && reinterpret_cast<uintptr_t>(workspace) % kWorkAlign == 0), "the workspace is NULL or not 16-byte aligned");
    if (!a.rows) return;
    a.num_sms = current_sms();
    a.most_rows = cache_attn_rows(a.bits, a.heads / a.kv_heads, max_new);
    a.blocks = cache_attn_blocks(a.bits, a.most_rows, a.num_sms);
    need(a.whole || workspace_bytes >= cache_attn_workspace(a.dim, a.most_rows, a.blocks), "the workspace is too small");
    a.work = static_cast<uint8_t*>(workspace);
    cuda(launch_cache_attn(a, static_cast<cudaStream_t>(stream)), "sync_cache_attn");
  });
}

}  // extern "C"

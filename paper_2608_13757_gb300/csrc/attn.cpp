// C ABI of the attention block's operators (include/sync.h): argument checks,
// plans of packed batches, and the launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <initializer_list>
#include <map>
#include <memory>
#include <mutex>
#include <new>
#include <queue>
#include <set>
#include <string>
#include <utility>
#include <vector>

#include "abi.h"
#include "attn.h"
#include "norm.h"

using namespace syncgb;
using namespace syncgb::abi;

namespace {

// ---- norm and rotation ----------------------------------------------------

void check_norm(const sync_norm_rope* p) {
  need(p, "the description must not be NULL");
  need(p->dtype == SYNC_BF16 || p->dtype == SYNC_FP16 || p->dtype == SYNC_FP32, "dtype must be a sync_dtype");
  need(p->heads >= 1 && p->kv_heads >= 1 && (int64_t)p->heads + p->kv_heads <= INT32_MAX / 256, "heads and kv_heads must be at least 1");
  need(p->dim >= 2 && p->dim <= 256 && p->dim % 2 == 0, "dim must be even and in 2..256");
  need(p->rotated >= 0 && p->rotated <= p->dim && p->rotated % 2 == 0, "rotated must be even and in 0..dim");
  need(std::isfinite(p->eps) && p->eps > 0.f, "eps must be positive and finite");
  need(p->q.rows >= 0 && p->q.rows == p->k.rows, "q and k must have the same number of rows");
  need(p->q.rows <= INT32_MAX, "more than INT32_MAX rows");
}

int entry_size(const sync_norm_rope* p) { return p->dtype == SYNC_FP32 ? 4 : 2; }

NormTensor norm_tensor(const sync_rows* t, const sync_norm_rope* p, const char* what) {
  need(t, what);
  need(t->rows == p->q.rows, "every tensor must have the rows of q");
  need(t->data || t->rows == 0, what);
  need_aligned(t->data, entry_size(p), "a tensor is not aligned to its type");
  NormTensor r;
  r.data = t->data;
  r.row = t->row_stride;
  r.head = t->head_stride;
  return r;
}

// Inputs may repeat a row or a head (a stride of 0); outputs may not, since
// warps in no order would write it.
NormTensor norm_output(const sync_rows* t, const sync_norm_rope* p, int32_t heads, const char* what) {
  const NormTensor r = norm_tensor(t, p, what);
  need((t->rows <= 1 || r.row) && (heads <= 1 || r.head), "an output's rows and heads must not share memory");
  return r;
}

NormArgs norm_args(const sync_norm_rope* p) {
  NormArgs a;
  need(p->rotated == 0 || p->q.rows == 0 || (p->cos && p->sin), "cos and sin must not be NULL");
  need(p->n_positions >= 0, "n_positions must not be negative");
  need_aligned(p->q_weight, entry_size(p), "q_weight is not aligned to its type");
  need_aligned(p->k_weight, entry_size(p), "k_weight is not aligned to its type");
  need_aligned(p->cos, 4, "cos is not aligned to its type");
  need_aligned(p->sin, 4, "sin is not aligned to its type");
  need_aligned(p->positions, 4, "positions is not aligned to its type");
  a.dtype = p->dtype;
  a.heads = p->heads;
  a.kv_heads = p->kv_heads;
  a.dim = p->dim;
  a.rotated = p->rotated;
  a.interleaved = p->interleaved != 0;
  a.eps = p->eps;
  a.inv_dim = 1.f / (float)p->dim;
  a.rows = p->q.rows;
  a.n_positions = p->n_positions;
  a.q = norm_tensor(&p->q, p, "q must not be NULL");
  a.k = norm_tensor(&p->k, p, "k must not be NULL");
  a.q_weight = p->q_weight;
  a.k_weight = p->k_weight;
  a.cos = p->cos;
  a.sin = p->sin;
  a.positions = p->positions;
  return a;
}

int64_t norm_workspace(const sync_norm_rope* p, int num_sms) {
  return (int64_t)norm_blocks(num_sms) * 2 * p->dim * (int64_t)sizeof(float);
}

// ---- attention ------------------------------------------------------------

void check_attn(const sync_attn_desc* d) {
  need(d, "the description must not be NULL");
  need(d->n_seqs >= 0, "n_seqs must not be negative");
  need(d->n_seqs == 0 || (d->q_len && d->k_len), "q_len and k_len must not be NULL");
  need(d->heads >= 1 && d->kv_heads >= 1 && d->heads % d->kv_heads == 0 && d->heads <= 65536, "heads must be a positive multiple of kv_heads, at most 65536");
  need(d->head_dim >= 8 && d->head_dim <= 128 && d->head_dim % 8 == 0, "head_dim must be a multiple of 8 in 8..128");
  need(d->dtype == SYNC_BF16 || d->dtype == SYNC_FP16, "dtype must be SYNC_BF16 or SYNC_FP16");
}

struct AttnSeq {
  int64_t q0, k0;                  // first rows in the query and key tensors
  int32_t lq, lk;
};

// Queries see the keys of their sequence up to their own place, or (not
// causal) all of them.
std::vector<AttnSeq> sequences(const sync_attn_desc* d, bool causal, sync_attn_sizes& sz) {
  std::vector<AttnSeq> seq((size_t)d->n_seqs);
  int64_t q = 0, k = 0;
  for (int32_t i = 0; i < d->n_seqs; ++i) {
    AttnSeq& s = seq[(size_t)i];
    const std::string where = "sequence " + std::to_string(i);
    s.lq = d->q_len[i];
    s.lk = d->k_len[i];
    if (s.lq < 0 || s.lk < 0) fail(SYNC_ERR_ARG, where + ": negative length");
    s.q0 = d->q_start ? d->q_start[i] : q;
    s.k0 = d->k_start ? d->k_start[i] : k;
    if (s.q0 < 0 || s.k0 < 0) fail(SYNC_ERR_ARG, where + ": negative start");
    if (s.q0 > INT32_MAX - (int64_t)s.lq || s.k0 > INT32_MAX - (int64_t)s.lk)
      fail(SYNC_ERR_OVERFLOW, where + ": rows past INT32_MAX");
    q = s.q0 + s.lq;
    k = s.k0 + s.lk;
    if (s.lq) sz.q_rows = std::max(sz.q_rows, q);
    if (s.lk) sz.k_rows = std::max(sz.k_rows, k);
    sz.n_queries += s.lq;
    sz.n_keys += s.lk;
    const int64_t seeing = std::min(s.lq, s.lk);
    sz.pairs += causal ? seeing * (s.lk - seeing) + seeing * (seeing + 1) / 2 : (int64_t)s.lq * s.lk;
  }
  // ranges of rows that are written must be disjoint
  auto disjoint = [&](int64_t AttnSeq::*start, int32_t AttnSeq::*len, const char* what) {
    std::vector<std::pair<int64_t, int64_t>> r;
    for (const AttnSeq& s : seq)
      if (s.*len) r.emplace_back(s.*start, s.*start + s.*len);
    std::sort(r.begin(), r.end());
    for (size_t i = 1; i < r.size(); ++i)
      if (r[i].first < r[i - 1].second) fail(SYNC_ERR_MALFORMED, what);
  };
  disjoint(&AttnSeq::q0, &AttnSeq::lq, "query ranges overlap");
  if (d->train) disjoint(&AttnSeq::k0, &AttnSeq::lk, "key ranges overlap in a plan with train set");
  return seq;
}

AttnTensor attn_tensor(const sync_rows* t, int64_t rows, const char* what) {
  need(t, what);
  need(t->rows >= rows && t->rows <= INT32_MAX, "a tensor has fewer rows than the plan needs, or more than INT32_MAX");
  need(t->data || rows == 0, what);
  need(reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->row_stride % 8 == 0 && t->head_stride % 8 == 0,
       "attention tensors must be 16-byte aligned with strides that are multiples of 8 entries");
  need(t->rows == 0 || (t->row_stride > 0 && t->head_stride > 0 && t->row_stride < (1ll << 38) && t->head_stride < (1ll << 38)),
       "strides must be positive and below 2^38 entries");
  AttnTensor r;
  r.data = t->data;
  r.rows = t->rows;
  r.row = t->row_stride;
  r.head = t->head_stride;
  return r;
}

auto encode_tiled() {
  static const auto f = driver_function<decltype(&cuTensorMapEncodeTiled)>("cuTensorMapEncodeTiled", 12000);
  if (!f) fail(SYNC_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  return f;
}

// Boxes of 64 entries, box_heads heads and box_rows rows; entries past the
// head's end and rows past the tensor's read as zero.
CUtensorMap tile_map(const AttnTensor& t, bool bf16, int heads, int dim, int box_heads, int box_rows) {
  CUtensorMap m;
  const cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)t.rows};
  const cuuint64_t stride[2] = {2ull * (cuuint64_t)t.head, 2ull * (cuuint64_t)t.row};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, one[3] = {1, 1, 1};
  const CUresult e = encode_tiled()(&m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, t.data,
                                    size, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (e != CUDA_SUCCESS) fail(SYNC_ERR_ARG, "a tensor's strides or address have no tile map (error " + std::to_string(e) + ")");
  return m;
}

// A sequence whose heads fill query tiles badly packs the heads of a group
// into one tile (128 / group queries each) where that takes fewer tiles.
bool packs(const AttnSeq& s, int group) {
  if (group == 1 || group > kTile) return false;
  const int64_t per = kTile / group;
  return (s.lq + per - 1) / per < (int64_t)group * ((s.lq + kTile - 1) / kTile);
}

// Plans of queries that see all keys go to the kernel of few queries (k_cache_attn.cu)
// where a key head's queries fit in 16 of its columns, or 8 in heads of more than
// 64 entries: it reads what there is and no more.  us there and in tiles of 128
// queries, bf16; n x m: n sequences of 1 to m keys, evenly drawn (one: m).  Up to 12
// sets of keys and values, 500 MB where 12 are enough for it, are taken in turn, so that
// they come from memory but for 4 x 100 and 16/2 heads at 300 x 100 and 16 x 1500:
//                              4 x 100  300 x 100  16 x 1500  48 x 1500   300 x 300  16 x 10000  1 x 100000
//   20 heads of 64, 1 query    6.8 6.2  25.2 93.6  17.1 20.5  39.0 49.1   52.4 120.8  78.7 92.5   89.3 102.8
//                 16 queries   7.9 6.0  32.7 93.6  23.4 20.3  48.1 49.3   70.0 120.6  87.2 92.9   92.8 104.0
//   16/2 heads of 64, 2        7.9 6.0   9.6 13.2  12.4 10.3  14.9 15.9   19.6  17.5  18.2 19.6   21.7  30.1
//   32/8 heads of 128, 1       7.8 6.6  18.3 49.6  15.5 18.3  32.4 30.3   45.0  64.5  61.3 59.5   69.1  73.4
//                      2       8.1 6.6  18.9 49.8  16.6 18.3  33.9 30.4   47.5  65.1  62.5 60.8   70.4  75.6
// The rule looks at rows and entries alone, and so takes the slower one in places: by
// 1 to 2.5 us of 6 where all tiles are one wave of blocks on up to 128 keys, by up to
// 27% with 9 to 16 rows in a few hundred passes or less, and by up to 20% in heads of
// more than 64 entries with hundreds of passes.  Tiles are up to three
// times as slow where sequences are many and short.  (16 rows of 128 entries, in a
// form that is gone: 48 x 1500 keys 38.4 against 28.2, 300 x 300 55.8 against 64.1.)
int64_t few_rows(int dim) { return dim <= 64 ? 16 : 8; }
bool few_queries(const sync_attn_desc* d, bool causal, const std::vector<AttnSeq>& seq) {
  if (causal || d->train || seq.empty() || seq.size() > (1u << 20)) return false;
  int64_t most = 0;
  for (const AttnSeq& s : seq) most = std::max<int64_t>(most, s.lq);
  return most > 0 && most * (d->heads / d->kv_heads) <= few_rows(d->head_dim);
}

// The longest of a plan's lists, before pieces are cut: what it would take to lay
// them out is known before anything is allocated for them.
int64_t longest_list(const sync_attn_desc* d, bool few, const std::vector<AttnSeq>& seq) {
  const int group = d->heads / d->kv_heads;
  int64_t items = 0, q = 0, k = 0;
  for (const AttnSeq& s : seq) {
    const bool packed = packs(s, group);
    const int64_t per = packed ? kTile / group : kTile;
    if (few) items += s.lq ? d->kv_heads : 0;
    else items += (s.lq + 2 * per - 1) / (2 * per) * (packed ? d->kv_heads : d->heads);
    if (!d->train) continue;
    q += (s.lq + kTile - 1ll) / kTile * d->heads;
    k += (s.lk + kTile - 1ll) / kTile * d->kv_heads;
  }
  return std::max(items, std::max(q, k));
}

struct ForwardWork {
  std::vector<AttnItem> item;
  std::vector<int32_t> block_first;
  std::vector<AttnSplit> split;
  int32_t slots = 0, merge_rows = 0;
};

// Items of a forward call and which block takes which.  An item's cost is the
// key tiles that its query tiles meet and kItemCost for what it does besides
// (a tile of one query tile takes about 0.8 us, an item's start and end 1.5).
constexpr int64_t kItemCost = 4, kMinPiece = 2;

template <class T>
struct Draft {
  T it;
  int64_t cost;
};

// The drafts in the order of the blocks that take them: from the most
// expensive on, always to the block that has least.  Returns the most that a
// block has.
template <class T>
int64_t assign(std::vector<Draft<T>>& all, int num_sms, std::vector<T>& item, std::vector<int32_t>& first) {
  std::stable_sort(all.begin(), all.end(), [](const Draft<T>& x, const Draft<T>& y) { return x.cost > y.cost; });
  const int blocks = (int)std::min<int64_t>(num_sms, (int64_t)all.size());
  std::vector<std::vector<int32_t>> of((size_t)blocks);
  using Load = std::pair<int64_t, int32_t>;
  std::priority_queue<Load, std::vector<Load>, std::greater<Load>> least;
  for (int32_t b = 0; b < blocks; ++b) least.push({0, b});
  int64_t most = 0;
  for (size_t i = 0; i < all.size(); ++i) {
    Load l = least.top();
    least.pop();
    of[(size_t)l.second].push_back((int32_t)i);
    l.first += all[i].cost;
    most = std::max(most, l.first);
    least.push(l);
  }
  first.push_back(0);
  for (const auto& b : of) {
    for (int32_t i : b) item.push_back(all[(size_t)i].it);
    first.push_back((int32_t)item.size());
  }
  return most;
}

// The items (most expensive first) on blocks that take `most` each: whole on
// the block that it fills best, or, where it fits nowhere, as much of it as the
// emptiest block has room for, and the rest likewise.  False if it does not fit.
bool cut(const std::vector<Draft<AttnItem>>& all, int group, int num_sms, int64_t most, ForwardWork& w) {
  w = ForwardWork{};
  std::vector<std::vector<AttnItem>> of((size_t)num_sms);
  std::set<std::pair<int64_t, int32_t>> rooms;                 // (room, -block): the first of equal ones is the last
  for (int32_t b = num_sms - 1; b >= 0; --b) rooms.emplace_hint(rooms.end(), most, -b);
  for (const Draft<AttnItem>& x : all) {
    const int32_t n = std::max(x.it.n[0], x.it.n[1]), slot0 = w.slots;
    auto cost = [&](int32_t a, int32_t b) {                    // of key tiles [a, b)
      int64_t c = kItemCost;
      for (int t = 0; t < 2; ++t) c += std::max(0, std::min(x.it.n[t], b) - std::min(x.it.n[t], a));
      return c;
    };
    int32_t from = 0;
    do {
      int32_t to = n;
      auto at = rooms.lower_bound({cost(from, n), -num_sms});
      if (at == rooms.end()) {
        at = std::prev(at);
        to = (int32_t)std::min(n - kMinPiece, from + at->first - kItemCost);       // a tile costs 1 or 2
        while (to > from && cost(from, to) > at->first) --to;
        if (to - from < kMinPiece) return false;
      }
      AttnItem it = x.it;
      it.k_row += (int64_t)from * kTile;
      it.seen -= from * kTile;
      it.keys -= from * kTile;
      for (int t = 0; t < 2; ++t) it.n[t] = std::max(0, std::min(x.it.n[t], to) - from);
      if (from > 0 || to < n) it.slot = w.slots++;
      auto room = rooms.extract(at);
      room.value().first -= cost(from, to);
      of[(size_t)-room.value().second].push_back(it);
      rooms.insert(std::move(room));
      from = to;
    } while (from < n);
    if (w.slots == slot0) continue;
    w.split.push_back({x.it.q_row, x.it.head, x.it.packed, {x.it.rows[0], x.it.rows[1]}, slot0, w.slots - slot0});
    w.merge_rows = std::max(w.merge_rows, (x.it.rows[0] + x.it.rows[1]) * (x.it.packed ? group : 1));
  }
  w.block_first.push_back(0);
  for (const auto& b : of) {
    if (b.empty()) continue;
    w.item.insert(w.item.end(), b.begin(), b.end());
    w.block_first.push_back((int32_t)w.item.size());
  }
  return true;
}

ForwardWork forward_work(const sync_attn_desc* d, bool causal, const std::vector<AttnSeq>& seq, int num_sms) {
  const int group = d->heads / d->kv_heads;
  std::vector<Draft<AttnItem>> draft;
  int64_t total = 0;
  for (const AttnSeq& s : seq) {
    const bool packed = packs(s, group);
    const int32_t per = packed ? kTile / group : kTile;
    for (int32_t h = 0; h < d->heads; h += packed ? group : 1)
      for (int64_t q0 = 0; q0 < s.lq; q0 += 2 * per) {
        AttnItem it{};
        it.q_row = s.q0 + q0;
        it.k_row = s.k0;
        it.head = h;
        it.packed = packed;
        it.seen = causal ? (int32_t)(q0 + s.lk - s.lq + 1) : s.lk;
        it.keys = s.lk;
        it.slot = -1;
        for (int t = 0; t < 2; ++t) {
          it.rows[t] = (int32_t)std::max<int64_t>(0, std::min<int64_t>(per, s.lq - q0 - t * per));
          const int64_t most = std::min<int64_t>((int64_t)it.seen + t * per + it.rows[t] - 1, s.lk);   // keys that the last query sees
          it.n[t] = it.rows[t] && most > 0 ? (int32_t)((most + kTile - 1) / kTile) : 0;
        }
        draft.push_back({it, it.n[0] + it.n[1] + kItemCost});
        total += draft.back().cost;
      }
  }
  ForwardWork w, whole;
  const int64_t most = assign(draft, num_sms, whole.item, whole.block_first);
  const int64_t share = std::max((total + num_sms - 1) / num_sms, kMinPiece + kItemCost);
  // Whole items balance well where there are many.  Where the fullest block
  // has 1/16 more than its share, items are cut along their keys and their
  // pieces' results merged: the least room per block in which they fit, if that
  // saves what the merge's launch takes.  A cut costs a write and a read of the
  // item's rows in 32 bits, so only what fits nowhere whole is cut (with every
  // block filled to its share, 151 cuts instead of 36, 5 prompts of 1535 tokens
  // behind 0-4099 keys took 57 us; 48 this way, 60 without cuts; 64 decode
  // steps over caches of 1-8096 keys 67, 64 and 78).
  for (int64_t room = share; room + std::max(kItemCost, room / 16) < most; room += room / 32 + 1)
    if (cut(draft, group, num_sms, room, w)) return w;
  return whole;
}

// Tiles of the gradients' two walks: key tiles with the query tiles that see
// them, over all heads of their group, and query tiles with the keys they see.
// These are not cut: the fullest block of the key walk has at least the steps of the
// first key tile of the longest sequence, for the whole group, which leaves SMs idle
// where key tiles and key heads are few (8192 tokens, 16 heads on 1 key head:
// 1024 steps where the mean is 219, a gradient of 1.47 ms against 0.86 on 2).
void gradient_work(const sync_attn_desc* d, bool causal, const std::vector<AttnSeq>& seq, std::vector<Draft<AttnTile>>& q,
                   std::vector<Draft<AttnTile>>& k) {
  const int64_t group = d->heads / d->kv_heads;
  for (const AttnSeq& s : seq) {
    const int64_t tiles = (s.lq + kTile - 1) / kTile, offset = (int64_t)s.lk - s.lq;
    AttnTile it{};
    for (int32_t h = 0; h < d->heads; ++h)
      for (int64_t q0 = 0; q0 < s.lq; q0 += kTile) {
        const int64_t most = causal ? std::min<int64_t>(q0 + kTile, s.lq) + offset : s.lk;       // keys that the last query sees
        it.q_row = s.q0 + q0;
        it.k_row = s.k0;
        it.head = h;
        it.n = (int32_t)(most > 0 ? (most + kTile - 1) / kTile : 0);
        it.rows = (int32_t)(s.lq - q0);
        it.keys = s.lk;
        it.seen = causal ? (int32_t)(q0 + offset + 1) : s.lk;
        q.push_back({it, it.n + kItemCost});
      }
    for (int32_t h = 0; h < d->kv_heads; ++h)
      for (int64_t k0 = 0; k0 < s.lk; k0 += kTile) {
        const int64_t first = causal ? std::min(tiles, std::max<int64_t>(0, k0 - offset) / kTile) : 0;   // the first tile that sees key k0
        it.q_row = s.q0 + first * kTile;
        it.k_row = s.k0 + k0;
        it.head = h;
        it.n = (int32_t)(tiles - first);
        it.rows = (int32_t)(s.lq - first * kTile);
        it.keys = (int32_t)(s.lk - k0);
        it.seen = causal ? (int32_t)(first * kTile + offset + 1 - k0) : kTile;   // (all of the tile)
        k.push_back({it, it.n * group + kItemCost});
      }
  }
}

// Device memory of a plan, laid out first, then allocated and filled at once.
class Arena {
 public:
  template <class T>
  size_t add(const std::vector<T>& v) {
    const size_t at = reserve(v.size() * sizeof(T));
    if (!v.empty()) {
      host_.resize(at + v.size() * sizeof(T));
      std::memcpy(host_.data() + at, v.data(), v.size() * sizeof(T));
    }
    return at;
  }
  size_t reserve(size_t bytes) {      // after every add(): not filled
    const size_t at = (size_ + 255) / 256 * 256;
    size_ = at + bytes;
    return at;
  }
  size_t size() const { return size_; }
  const std::vector<uint8_t>& host() const { return host_; }

 private:
  size_t size_ = 0;
  std::vector<uint8_t> host_;
};

// Copies to the device on a stream of the library's own and waits for that
// stream alone: the copy is complete for kernels on any stream, and the
// caller's queued work is not waited for.
void upload(int device, void* to, const void* from, size_t bytes) {
  static std::mutex mu;
  static std::map<int, cudaStream_t> streams;
  cudaStream_t st = nullptr;
  {
    std::lock_guard<std::mutex> lock(mu);
    auto at = streams.find(device);
    if (at == streams.end()) {
      cuda(cudaStreamCreateWithFlags(&st, cudaStreamNonBlocking), "cudaStreamCreate");
      streams.emplace(device, st);
    } else {
      st = at->second;
    }
  }
  cuda(cudaMemcpyAsync(to, from, bytes, cudaMemcpyHostToDevice, st), "sync_attn_plan");
  cuda(cudaStreamSynchronize(st), "sync_attn_plan");
}

void check_gave_up(const sync_attn* plan) {
  if (*static_cast<volatile int*>(plan->error))
    fail(SYNC_ERR_CUDA, "a call on this plan gave up waiting inside a kernel: its results are not valid");
}

}  // namespace

// For tests on the host: the work lists of a plan for a GPU of num_sms SMs,
// one row of `width` values per item.  which 0: forward items (block, q_row,
// k_row, head, packed, rows of both tiles, key tiles of both, seen, keys,
// slot); 1: split ranges (q_row, head, packed, rows of both, slot, pieces);
// 2 and 3: query and key tiles of the gradients (block, q_row, k_row, head, n,
// rows, keys, seen).  Returns the rows (written up to `capacity`), or a
// negative status.
static int64_t work_rows(const sync_attn_desc* desc, bool causal, int num_sms, int which, int64_t* out, int64_t capacity) {
  int64_t n = 0;
  const sync_status status = guarded([&] {
    check_attn(desc);
    sync_attn_sizes sz{};
    const std::vector<AttnSeq> seq = sequences(desc, causal, sz);
    auto row = [&](std::initializer_list<int64_t> v) {
      if (n < capacity) std::copy(v.begin(), v.end(), out + n * (int64_t)v.size());
      ++n;
    };
    if (which < 2) {
      const ForwardWork w = forward_work(desc, causal, seq, num_sms);
      if (which == 1) {
        for (const AttnSplit& s : w.split) row({s.q_row, s.head, s.packed, s.rows[0], s.rows[1], s.slot, s.pieces});
        return;
      }
      for (size_t b = 0; b + 1 < w.block_first.size(); ++b)
        for (int32_t i = w.block_first[b]; i < w.block_first[b + 1]; ++i) {
          const AttnItem& x = w.item[(size_t)i];
          row({(int64_t)b, x.q_row, x.k_row, x.head, x.packed, x.rows[0], x.rows[1], x.n[0], x.n[1], x.seen, x.keys, x.slot});
        }
      return;
    }
    std::vector<Draft<AttnTile>> q, k;
    gradient_work(desc, causal, seq, q, k);
    std::vector<AttnTile> tile;
    std::vector<int32_t> first;
    assign(which == 2 ? q : k, num_sms, tile, first);
    for (size_t b = 0; b + 1 < first.size(); ++b)
      for (int32_t i = first[b]; i < first[b + 1]; ++i) {
        const AttnTile& x = tile[(size_t)i];
        row({(int64_t)b, x.q_row, x.k_row, x.head, x.n, x.rows, x.keys, x.seen});
      }
  });
  return status == SYNC_OK ? n : -(int64_t)status;
}
extern "C" int64_t syncgb_attn_work(const sync_attn_desc* desc, int num_sms, int which, int64_t* out, int64_t capacity) {
  return work_rows(desc, true, num_sms, which, out, capacity);
}
extern "C" int64_t syncgb_cross_attn_work(const sync_attn_desc* desc, int num_sms, int which, int64_t* out, int64_t capacity) {
  return work_rows(desc, false, num_sms, which, out, capacity);
}

// For tests: a kernel of the plan whose waits run out after `tries` tries.
extern "C" sync_status syncgb_attn_wait_in_vain(const sync_attn* plan, int tries, void* stream) {
  return guarded([&] {
    need(plan && tries >= 1, "plan must not be NULL, tries at least 1");
    DeviceScope scope(plan->device);
    cuda(launch_wait_in_vain(plan->error, tries, static_cast<cudaStream_t>(stream)), "syncgb_attn_wait_in_vain");
  });
}

extern "C" {

sync_status sync_qk_norm_rope(const sync_norm_rope* p, const sync_rows* q_out, const sync_rows* k_out, void* stream) {
  return guarded([&] {
    check_norm(p);
    NormArgs a = norm_args(p);
    a.q_out = norm_output(q_out, p, p->heads, "q_out must not be NULL");
    a.k_out = norm_output(k_out, p, p->kv_heads, "k_out must not be NULL");
    a.num_sms = current_sms();
    cuda(launch_norm_rope(a, static_cast<cudaStream_t>(stream)), "sync_qk_norm_rope");
  });
}

sync_status sync_qk_norm_rope_workspace(const sync_norm_rope* p, int64_t* bytes) {
  return guarded([&] {
    check_norm(p);
    need(bytes, "bytes must not be NULL");
    *bytes = norm_workspace(p, current_sms());
  });
}

sync_status sync_qk_norm_rope_backward(const sync_norm_rope* p, const sync_rows* dq_out, const sync_rows* dk_out,
                                       const sync_rows* dq, const sync_rows* dk, void* dq_weight, void* dk_weight,
                                       void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&] {
    check_norm(p);
    NormArgs a = norm_args(p);
    a.grad = true;
    a.q_out = norm_tensor(dq_out, p, "dq_out must not be NULL");
    a.k_out = norm_tensor(dk_out, p, "dk_out must not be NULL");
    a.dq = norm_output(dq, p, p->heads, "dq must not be NULL");
    a.dk = norm_output(dk, p, p->kv_heads, "dk must not be NULL");
    need(!p->q_weight == !dq_weight && !p->k_weight == !dk_weight, "a weight and its gradient must both be given or both be NULL");
    need_aligned(dq_weight, entry_size(p), "dq_weight is not aligned to its type");
    need_aligned(dk_weight, entry_size(p), "dk_weight is not aligned to its type");
    a.num_sms = current_sms();
    need(workspace && workspace_bytes >= norm_workspace(p, a.num_sms) && reinterpret_cast<uintptr_t>(workspace) % 16 == 0,
         "the workspace is NULL, too small or not 16-byte aligned");
    a.q_weight_grad = dq_weight;
    a.k_weight_grad = dk_weight;
    a.partial = static_cast<float*>(workspace);
    cuda(launch_norm_rope(a, static_cast<cudaStream_t>(stream)), "sync_qk_norm_rope_backward");
  });
}

static sync_status make_plan(const sync_attn_desc* desc, bool causal, int device, sync_attn** out) {
  return guarded([&] {
    need(out, "out must not be NULL");
    *out = nullptr;
    check_attn(desc);
    sync_attn_sizes sz{};
    const std::vector<AttnSeq> seq = sequences(desc, causal, sz);
    const bool few = few_queries(desc, causal, seq);
    if (longest_list(desc, few, seq) > INT32_MAX) fail(SYNC_ERR_OVERFLOW, "more than INT32_MAX work items");
    DeviceScope scope(device);
    std::unique_ptr<sync_attn, void (*)(sync_attn*)> P(new sync_attn, sync_attn_free);
    P->device = device;
    P->num_sms = sm_count(device);
    P->train = desc->train != 0;
    AttnArgs& a = P->args;
    a.bf16 = desc->dtype == SYNC_BF16;
    a.heads = desc->heads;
    a.kv_heads = desc->kv_heads;
    a.dim = desc->head_dim;
    a.num_sms = P->num_sms;
    P->few = few;
    std::vector<int32_t> q_row, q_len, k_len;
    std::vector<int64_t> k_row;
    CacheArgs& f = P->rows;
    if (P->few) {
      int32_t most_q = 0, most_k = 0;
      for (const AttnSeq& s : seq) {
        if (s.lq == 0) continue;
        q_row.push_back((int32_t)s.q0);
        q_len.push_back(s.lq);
        k_len.push_back(s.lk);
        k_row.push_back(s.k0);
        most_q = std::max(most_q, s.lq);
        most_k = std::max(most_k, s.lk);
      }
      f.bf16 = a.bf16;
      f.heads = a.heads;
      f.kv_heads = a.kv_heads;
      f.dim = a.dim;
      f.n_seqs = (int)q_row.size();
      f.num_sms = P->num_sms;
      f.most_rows = cache_attn_rows(16, a.heads / a.kv_heads, most_q);
      f.blocks = cache_attn_blocks(16, f.most_rows, P->num_sms);
      f.whole = most_k <= SYNC_CACHE_SHORT;
    }
    const ForwardWork w = P->few ? ForwardWork{} : forward_work(desc, causal, seq, P->num_sms);
    a.n_blocks = std::max<int>(0, (int)w.block_first.size() - 1);
    std::vector<AttnTile> qt, kt;
    std::vector<int32_t> q_first, k_first;
    if (P->train) {
      std::vector<Draft<AttnTile>> q, k;
      gradient_work(desc, causal, seq, q, k);
      assign(q, P->num_sms, qt, q_first);
      assign(k, P->num_sms, kt, k_first);
      a.n_q_blocks = (int)q_first.size() - 1;
      a.n_k_blocks = (int)k_first.size() - 1;
    }
    a.delta_rows = sz.q_rows;
    Arena m;
    const size_t at_item = m.add(w.item), at_first = m.add(w.block_first), at_split = m.add(w.split),
                 at_qt = m.add(qt), at_kt = m.add(kt), at_qf = m.add(q_first), at_kf = m.add(k_first),
                 at_row = m.add(q_row), at_len = m.add(q_len), at_keys = m.add(k_len), at_key = m.add(k_row);
    const size_t padded = a.dim <= 64 ? 64 : 128;
    const size_t at_part = m.reserve((size_t)w.slots * 2 * kTile * padded * sizeof(float)),
                 at_part_lse = m.reserve((size_t)w.slots * 2 * kTile * sizeof(float)),
                 at_delta = m.reserve(P->train ? (size_t)sz.q_rows * (size_t)a.heads * sizeof(float) : 0);
    const size_t at_work = m.reserve(P->few && !f.whole ? (size_t)cache_attn_workspace(a.dim, f.most_rows, f.blocks) : 0);
    cuda(cudaMallocHost(reinterpret_cast<void**>(&P->error), sizeof(int)), "sync_attn_plan");
    *P->error = 0;
    a.error = P->error;
    cuda(cudaMalloc(&P->block, std::max<size_t>(m.size(), 1)), "sync_attn_plan");
    upload(device, P->block, m.host().data(), m.host().size());
    uint8_t* base = static_cast<uint8_t*>(P->block);
    a.item = reinterpret_cast<const AttnItem*>(base + at_item);
    a.block_first = reinterpret_cast<const int32_t*>(base + at_first);
    a.split = reinterpret_cast<const AttnSplit*>(base + at_split);
    a.n_splits = (int)w.split.size();
    a.merge_rows = w.merge_rows;
    a.q_tile = reinterpret_cast<const AttnTile*>(base + at_qt);
    a.k_tile = reinterpret_cast<const AttnTile*>(base + at_kt);
    a.q_first = reinterpret_cast<const int32_t*>(base + at_qf);
    a.k_first = reinterpret_cast<const int32_t*>(base + at_kf);
    a.part_o = reinterpret_cast<float*>(base + at_part);
    a.part_lse = reinterpret_cast<float*>(base + at_part_lse);
    a.delta = reinterpret_cast<float*>(base + at_delta);
    f.starts = reinterpret_cast<const int32_t*>(base + at_row);
    f.counts = reinterpret_cast<const int32_t*>(base + at_len);
    f.lens = reinterpret_cast<const int32_t*>(base + at_keys);
    f.firsts = reinterpret_cast<const int64_t*>(base + at_key);
    f.work = base + at_work;
    sz.device_bytes = (int64_t)m.size();
    sz.n_items = P->few ? f.n_seqs * a.kv_heads : (int32_t)w.item.size();
    sz.n_splits = w.slots;
    P->sz = sz;
    *out = P.release();
  });
}

sync_status sync_attn_plan(const sync_attn_desc* desc, int device, sync_attn** out) {
  return make_plan(desc, true, device, out);
}

sync_status sync_cross_attn_plan(const sync_attn_desc* desc, int device, sync_attn** out) {
  return make_plan(desc, false, device, out);
}

sync_status sync_attn_query(const sync_attn* plan, sync_attn_sizes* out) {
  return guarded([&] {
    need(plan && out, "plan and out must not be NULL");
    *out = plan->sz;
  });
}

sync_status sync_attn_status(const sync_attn* plan) {
  return guarded([&] {
    need(plan, "plan must not be NULL");
    check_gave_up(plan);
  });
}

sync_status sync_attn_forward(const sync_attn* plan, const sync_rows* q, const sync_rows* k, const sync_rows* v,
                              float scale, const sync_rows* o, float* lse, void* stream) {
  return guarded([&] {
    need(plan, "plan must not be NULL");
    need(std::isfinite(scale) && scale > 0.f, "scale must be positive and finite");
    need_aligned(lse, 4, "lse is not aligned to its type");
    AttnArgs a = plan->args;
    a.scale = scale;
    a.q = attn_tensor(q, plan->sz.q_rows, "q must not be NULL");
    a.k = attn_tensor(k, plan->sz.k_rows, "k must not be NULL");
    a.v = attn_tensor(v, plan->sz.k_rows, "v must not be NULL");
    a.o = attn_tensor(o, plan->sz.q_rows, "o must not be NULL");
    a.lse = lse;
    if (!a.n_blocks && !plan->few) return;
    check_gave_up(plan);
    DeviceScope scope(plan->device);
    if (plan->few) {
      auto rows = [](const AttnTensor& t) {
        HeadTensor r;
        r.data = t.data;
        r.rows = t.rows;
        r.row = t.row;
        r.head = t.head;
        return r;
      };
      CacheArgs f = plan->rows;
      f.rows = a.q.rows;
      f.scale = scale;
      f.q = rows(a.q);
      f.q_out = rows(a.o);
      f.k_rows = rows(a.k);
      f.v_rows = rows(a.v);
      f.lse = lse;
      cuda(launch_few_queries(f, static_cast<cudaStream_t>(stream)), "sync_attn_forward");
      return;
    }
    const int group = a.heads / a.kv_heads;
    AttnMaps m{};
    m.q = tile_map(a.q, a.bf16, a.heads, a.dim, 1, kTile);
    m.q_group = group > kTile ? m.q : tile_map(a.q, a.bf16, a.heads, a.dim, group, kTile / group);
    if (a.k.rows) {
      m.k = tile_map(a.k, a.bf16, a.kv_heads, a.dim, 1, kTile);
      m.v = tile_map(a.v, a.bf16, a.kv_heads, a.dim, 1, kTile);
    }
    cuda(launch_attn_forward(a, m, static_cast<cudaStream_t>(stream)), "sync_attn_forward");
  });
}

sync_status sync_attn_backward(const sync_attn* plan, const sync_rows* q, const sync_rows* k, const sync_rows* v,
                               const sync_rows* o, const float* lse, const sync_rows* d_o, float scale,
                               const sync_rows* dq, const sync_rows* dk, const sync_rows* dv, void* stream) {
  return guarded([&] {
    need(plan, "plan must not be NULL");
    need(plan->train, "the plan was made without train set");
    need(std::isfinite(scale) && scale > 0.f, "scale must be positive and finite");
    need(lse || plan->sz.q_rows == 0, "lse must not be NULL");
    need_aligned(lse, 4, "lse is not aligned to its type");
    AttnArgs a = plan->args;
    a.scale = scale;
    a.q = attn_tensor(q, plan->sz.q_rows, "q must not be NULL");
    a.k = attn_tensor(k, plan->sz.k_rows, "k must not be NULL");
    a.v = attn_tensor(v, plan->sz.k_rows, "v must not be NULL");
    a.o = attn_tensor(o, plan->sz.q_rows, "o must not be NULL");
    a.d_o = attn_tensor(d_o, plan->sz.q_rows, "d_o must not be NULL");
    a.dq = attn_tensor(dq, plan->sz.q_rows, "dq must not be NULL");
    a.dk = attn_tensor(dk, plan->sz.k_rows, "dk must not be NULL");
    a.dv = attn_tensor(dv, plan->sz.k_rows, "dv must not be NULL");
    a.lse = const_cast<float*>(lse);
    if (!a.n_q_blocks && !a.n_k_blocks) return;
    check_gave_up(plan);
    DeviceScope scope(plan->device);
    AttnMaps m{};
    if (a.q.rows) {
      m.q = tile_map(a.q, a.bf16, a.heads, a.dim, 1, kTile);
      m.d_o = tile_map(a.d_o, a.bf16, a.heads, a.dim, 1, kTile);
    }
    if (a.k.rows) {
      m.k = tile_map(a.k, a.bf16, a.kv_heads, a.dim, 1, kTile);
      m.v = tile_map(a.v, a.bf16, a.kv_heads, a.dim, 1, kTile);
    }
    cuda(launch_attn_backward(a, m, static_cast<cudaStream_t>(stream)), "sync_attn_backward");
  });
}

void sync_attn_free(sync_attn* plan) {
  if (!plan) return;
  int was = 0;
  const bool have = cudaGetDevice(&was) == cudaSuccess;
  cudaSetDevice(plan->device);
  cudaDeviceSynchronize();
  if (plan->block) cudaFree(plan->block);
  if (plan->error) cudaFreeHost(plan->error);
  if (have && was != plan->device) cudaSetDevice(was);
  delete plan;
}

}  // extern "C"

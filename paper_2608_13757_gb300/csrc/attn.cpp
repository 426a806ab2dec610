// C ABI of the attention block's operators (include/sync.h): argument checks,
// plans of packed batches, and the launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <numeric>
#include <string>
#include <utility>
#include <vector>

#include "attn.h"
#include "handle.h"
#include "norm.h"

using namespace syncgb;

namespace {

struct Failure {
  sync_status status;
  std::string msg;
};

[[noreturn]] void fail(sync_status s, std::string msg) { throw Failure{s, std::move(msg)}; }

void need(bool ok, const char* what) {
  if (!ok) fail(SYNC_ERR_ARG, what);
}

void cuda(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return;
  if (e == cudaErrorMemoryAllocation) cudaGetLastError();
  fail(e == cudaErrorMemoryAllocation ? SYNC_ERR_OOM : SYNC_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// Runs f with every failure turned into a status.
template <class F>
sync_status guarded(F&& f) {
  try {
    f();
    return SYNC_OK;
  } catch (const Failure& e) {
    return set_error(e.status, e.msg);
  } catch (const std::bad_alloc&) {
    return set_error(SYNC_ERR_OOM, "host allocation failed");
  } catch (...) {
    return set_error(SYNC_ERR_ARG, "unexpected error");
  }
}

// The device that a call works on, set for its duration.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    cuda(cudaGetDevice(&was_), "cudaGetDevice");
    if (was_ != device) cuda(cudaSetDevice(device), "cudaSetDevice");
    set_ = was_ != device;
  }
  ~DeviceScope() {
    if (set_) cudaSetDevice(was_);
  }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;

 private:
  int was_ = 0;
  bool set_ = false;
};

int sm_count(int device) {
  int n = 0;
  cuda(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device), "cudaDeviceGetAttribute");
  return n;
}

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

NormTensor norm_tensor(const sync_rows* t, const sync_norm_rope* p, const char* what) {
  need(t, what);
  need(t->rows == p->q.rows, "every tensor must have the rows of q");
  need(t->data || t->rows == 0, what);
  need(reinterpret_cast<uintptr_t>(t->data) % (p->dtype == SYNC_FP32 ? 4 : 2) == 0, "a tensor is not aligned to its type");
  NormTensor r;
  r.data = t->data;
  r.row = t->row_stride;
  r.head = t->head_stride;
  return r;
}

NormArgs norm_args(const sync_norm_rope* p) {
  NormArgs a;
  need(p->rotated == 0 || p->q.rows == 0 || (p->cos && p->sin), "cos and sin must not be NULL");
  need(p->n_positions >= 0, "n_positions must not be negative");
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
  int device = 0;
  cuda(cudaGetDevice(&device), "cudaGetDevice");
  a.num_sms = sm_count(device);
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

std::vector<AttnSeq> sequences(const sync_attn_desc* d, sync_attn_sizes& sz) {
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
    sz.pairs += seeing * (s.lk - seeing) + seeing * (seeing + 1) / 2;
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
  AttnTensor r;
  r.data = t->data;
  r.rows = t->rows;
  r.row = t->row_stride;
  r.head = t->head_stride;
  return r;
}

}  // namespace

extern "C" {

sync_status sync_qk_norm_rope(const sync_norm_rope* p, const sync_rows* q_out, const sync_rows* k_out, void* stream) {
  return guarded([&] {
    check_norm(p);
    NormArgs a = norm_args(p);
    a.q_out = norm_tensor(q_out, p, "q_out must not be NULL");
    a.k_out = norm_tensor(k_out, p, "k_out must not be NULL");
    cuda(launch_norm_rope(a, static_cast<cudaStream_t>(stream)), "sync_qk_norm_rope");
  });
}

sync_status sync_qk_norm_rope_workspace(const sync_norm_rope* p, int64_t* bytes) {
  return guarded([&] {
    check_norm(p);
    need(bytes, "bytes must not be NULL");
    int device = 0;
    cuda(cudaGetDevice(&device), "cudaGetDevice");
    *bytes = norm_workspace(p, sm_count(device));
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
    a.dq = norm_tensor(dq, p, "dq must not be NULL");
    a.dk = norm_tensor(dk, p, "dk must not be NULL");
    need(!p->q_weight == !dq_weight && !p->k_weight == !dk_weight, "a weight and its gradient must both be given or both be NULL");
    need(workspace && workspace_bytes >= norm_workspace(p, a.num_sms) && reinterpret_cast<uintptr_t>(workspace) % 16 == 0,
         "the workspace is NULL, too small or not 16-byte aligned");
    a.q_weight_grad = dq_weight;
    a.k_weight_grad = dk_weight;
    a.partial = static_cast<float*>(workspace);
    cuda(launch_norm_rope(a, static_cast<cudaStream_t>(stream)), "sync_qk_norm_rope_backward");
  });
}

sync_status sync_attn_plan(const sync_attn_desc* desc, int device, sync_attn** out) {
  return guarded([&] {
    need(out, "out must not be NULL");
    *out = nullptr;
    check_attn(desc);
    sync_attn_sizes sz{};
    const std::vector<AttnSeq> seq = sequences(desc, sz);
    std::vector<AttnItem> qi, ki;
    for (int32_t i = 0; i < desc->n_seqs; ++i) {
      for (int32_t h = 0; h < desc->heads; ++h)
        for (int32_t t = 0; t * kTile < seq[(size_t)i].lq; ++t) qi.push_back({i, h, t, 0});
      for (int32_t h = 0; h < desc->kv_heads; ++h)
        for (int32_t t = 0; t * kTile < seq[(size_t)i].lk; ++t) ki.push_back({i, h, t, 0});
    }
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
    auto put = [&](const auto& v) {
      using T = typename std::decay_t<decltype(v)>::value_type;
      void* d = nullptr;
      if (v.empty()) return static_cast<const T*>(nullptr);
      cuda(cudaMalloc(&d, v.size() * sizeof(T)), "sync_attn_plan");
      P->blocks.push_back(d);
      sz.device_bytes += (int64_t)(v.size() * sizeof(T));
      cuda(cudaMemcpy(d, v.data(), v.size() * sizeof(T), cudaMemcpyHostToDevice), "sync_attn_plan");
      return static_cast<const T*>(d);
    };
    a.seq = put(seq);
    a.q_item = put(qi);
    a.n_q_items = (int)qi.size();
    a.k_item = put(ki);
    a.n_k_items = (int)ki.size();
    if (P->train && sz.q_rows) {
      void* d = nullptr;
      const size_t bytes = (size_t)sz.q_rows * (size_t)a.heads * sizeof(float);
      cuda(cudaMalloc(&d, bytes), "sync_attn_plan");
      P->blocks.push_back(d);
      sz.device_bytes += (int64_t)bytes;
      a.delta = static_cast<float*>(d);
      a.delta_rows = sz.q_rows;
    }
    sz.n_items = a.n_q_items;
    P->sz = sz;
    *out = P.release();
  });
}

sync_status sync_attn_query(const sync_attn* plan, sync_attn_sizes* out) {
  return guarded([&] {
    need(plan && out, "plan and out must not be NULL");
    *out = plan->sz;
  });
}

sync_status sync_attn_forward(const sync_attn* plan, const sync_rows* q, const sync_rows* k, const sync_rows* v,
                              float scale, const sync_rows* o, float* lse, void* stream) {
  return guarded([&] {
    need(plan, "plan must not be NULL");
    need(std::isfinite(scale) && scale > 0.f, "scale must be positive and finite");
    AttnArgs a = plan->args;
    a.scale = scale;
    a.q = attn_tensor(q, plan->sz.q_rows, "q must not be NULL");
    a.k = attn_tensor(k, plan->sz.k_rows, "k must not be NULL");
    a.v = attn_tensor(v, plan->sz.k_rows, "v must not be NULL");
    a.o = attn_tensor(o, plan->sz.q_rows, "o must not be NULL");
    a.lse = lse;
    if (!a.n_q_items) return;
    DeviceScope scope(plan->device);
    cuda(launch_attn_forward(a, static_cast<cudaStream_t>(stream)), "sync_attn_forward");
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
    if (!a.n_q_items && !a.n_k_items) return;
    DeviceScope scope(plan->device);
    cuda(launch_attn_backward(a, static_cast<cudaStream_t>(stream)), "sync_attn_backward");
  });
}

void sync_attn_free(sync_attn* plan) {
  if (!plan) return;
  int was = 0;
  const bool have = cudaGetDevice(&was) == cudaSuccess;
  cudaSetDevice(plan->device);
  cudaDeviceSynchronize();
  for (void* b : plan->blocks) cudaFree(b);
  if (have && was != plan->device) cudaSetDevice(was);
  delete plan;
}

}  // extern "C"

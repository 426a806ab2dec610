// What the C calls of the operators share (attn.cpp, cache.cpp): failures as
// exceptions inside the library and as a status outside, and the device of a call.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <new>
#include <string>
#include <utility>

#include "handle.h"

namespace syncgb {
namespace abi {

struct Failure {
  sync_status status;
  std::string msg;
};

[[noreturn]] inline void fail(sync_status s, std::string msg) { throw Failure{s, std::move(msg)}; }

inline void need(bool ok, const char* what) {
  if (!ok) fail(SYNC_ERR_ARG, what);
}

inline void cuda(cudaError_t e, const char* what) {
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

// A function of the driver, or null.
template <class F>
F driver_function(const char* name, unsigned version) {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult r;
  if (cudaGetDriverEntryPointByVersion(name, &p, version, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess)
    p = nullptr;
  return reinterpret_cast<F>(p);
}

// Whether this thread has a context.  One that has made no call of the runtime
// yet has none (a framework's backward pass runs on such threads), and encoding
// a tile map needs one, which it does not make itself.
inline bool has_context() {
  static const auto f = driver_function<decltype(&cuCtxGetCurrent)>("cuCtxGetCurrent", 4000);
  CUcontext c = nullptr;
  return f && f(&c) == CUDA_SUCCESS && c;
}

// The device that a call works on, set for its duration.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    cuda(cudaGetDevice(&was_), "cudaGetDevice");
    set_ = was_ != device;
    if (set_ || !has_context()) cuda(cudaSetDevice(device), "cudaSetDevice");
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

inline int sm_count(int device) {
  int n = 0;
  cuda(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device), "cudaDeviceGetAttribute");
  return n;
}

inline int current_sms() {
  int device = 0;
  cuda(cudaGetDevice(&device), "cudaGetDevice");
  return sm_count(device);
}

// A pointer that is NULL or a multiple of its type's size.
inline void need_aligned(const void* p, int size, const char* what) {
  need(reinterpret_cast<uintptr_t>(p) % size == 0, what);
}

}  // namespace abi
}  // namespace syncgb

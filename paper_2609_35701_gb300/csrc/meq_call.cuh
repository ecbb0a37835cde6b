// What the stateless calls of the C ABI share: statuses, their texts, and checks
// of pointers.
#pragma once

#include <map>
#include <mutex>
#include <new>
#include <string>

#include "meq_internal.cuh"

namespace meq {

inline meq_status fail(meq_status s, const std::string& msg) {
  set_global_error(msg);
  return s;
}
inline meq_status launch_status(cudaError_t e, const char* fn, const char* what) {
  if (e == cudaSuccess) return MEQ_OK;
  return fail(MEQ_ERR_CUDA, std::string(fn) + ": " + what + ": " + cudaGetErrorString(e));
}
template <typename F>
meq_status guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return MEQ_ERR_OOM;
  } catch (...) {
    return MEQ_ERR_INVALID_ARG;
  }
}

inline bool valid_type(int type) { return type == MEQ_F32 || type == MEQ_BF16 || type == MEQ_F16; }
inline int elem_bytes(int type) { return type == MEQ_F32 ? 4 : 2; }

inline int device_sms(cudaError_t* e) {
  int dev = 0, sms = 0;
  *e = cudaGetDevice(&dev);
  if (*e == cudaSuccess) *e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

// Lets a kernel have more dynamic shared memory than 48 KB, once per device.
template <typename F>
cudaError_t allow_shared(F* kernel, int bytes) {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static std::map<const void*, uint64_t> known;  // a bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  uint64_t& bits = known[reinterpret_cast<const void*>(kernel)];
  if (!((bits >> dev) & 1)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    bits |= uint64_t(1) << dev;
  }
  return cudaSuccess;
}

inline bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace meq

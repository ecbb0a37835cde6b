// What the stateless calls of the C ABI share: statuses, their texts, and checks
// of pointers.
#pragma once

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

inline bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace meq

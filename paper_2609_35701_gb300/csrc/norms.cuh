// Arguments and shared pieces of the norms' kernels.
#pragma once

#include <cfloat>

#include "meq_elem.cuh"
#include "meq_elementwise.cuh"

namespace meq {
namespace norm {

struct ForwardArgs {
  const void* x;
  const void* residual;  // NULL: none
  const void* weight;    // NULL: 1
  const void* bias;      // NULL: 0
  void* y;
  void* h;               // x + residual; NULL without a residual
  float* mean;           // NULL: RMS norm
  float* rstd;
  int64_t rows, cols, ld_x, ld_residual, ld_y, ld_h;
  int weight_type;
  float eps;
};

struct BackwardArgs {
  const void* dy;
  const void* h;
  const void* dh;       // NULL: none
  const void* weight;   // NULL: 1
  const float* mean;    // NULL: RMS norm
  const float* rstd;
  void* dx;
  int64_t rows, cols, ld_dy, ld_h, ld_dh, ld_dx;
  int weight_type;
  float* parts;         // [2][parts][cols]: partial sums of dy xhat and of dy; NULL: they are not wanted
  void* dweight;        // launch_few_backward: the sums themselves; either may be NULL
  void* dbias;
  int grad_type;
  float* row_sums;      // wide rows: mean(a xhat) and mean(a) of each row
};

// Element i of an array of the given meq_dtype.
__device__ __forceinline__ float load_as(const void* p, int type, int64_t i) {
  if (type == MEQ_F32) return static_cast<const float*>(p)[i];
  if (type == MEQ_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int type, int64_t i, float x) {
  if (type == MEQ_F32) static_cast<float*>(p)[i] = x;
  else if (type == MEQ_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  else static_cast<__half*>(p)[i] = __float2half_rn(x);
}

// 1 / sqrt(var + eps) (an approximation and a Newton step: within 2^-24 or so),
// NaN where the sum of squares was not finite: a root of an infinity would make
// the row 0.
__device__ __forceinline__ float inverse_root(float var, float eps) {
  const float x = var + eps, r = rsqrtf(x);
  const float e = fmaf(-x * r, r, 1.f);
  return var <= FLT_MAX && x <= FLT_MAX ? fmaf(0.5f * r, e, r) : __int_as_float(0x7fc00000);
}

}  // namespace norm
}  // namespace meq

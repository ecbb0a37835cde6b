// Elements of the three types in 16-byte pieces, shared by the losses, the norms
// and the embedding.
#pragma once

#include <cmath>

#include "meq_internal.cuh"

namespace meq {

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNegInf = 0xFF800000u;
  static __device__ __forceinline__ void unpack(uint4 q, float2* x) {
    x[0] = make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
    x[1] = make_float2(__uint_as_float(q.z), __uint_as_float(q.w));
  }
  static __device__ __forceinline__ uint4 pack(const float2* x) {
    return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
  }
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  using Max = float;  // running maximum of the elements of pieces
  static __device__ __forceinline__ Max max_of(Max m, uint4 q) {
    return fmaxf(fmaxf(fmaxf(m, __uint_as_float(q.x)), fmaxf(__uint_as_float(q.y), __uint_as_float(q.z))), __uint_as_float(q.w));
  }
  static __device__ __forceinline__ Max none() { return -INFINITY; }
  static __device__ __forceinline__ float value(Max m) { return m; }
  using Bits = uint32_t;
  static __device__ __forceinline__ float make(float x) { return x; }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr uint32_t kNegInf = 0xFF80FF80u;
  static __device__ __forceinline__ void unpack(uint4 q, float2* x) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint4 pack(const float2* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[i].x, x[i].y);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  using Max = __nv_bfloat162;  // two at a time, without widening
  static __device__ __forceinline__ Max max_of(Max m, uint4 q) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
    return __hmax2(__hmax2(__hmax2(m, h[0]), __hmax2(h[1], h[2])), h[3]);
  }
  static __device__ __forceinline__ Max none() {
    const uint32_t w = kNegInf;
    return *reinterpret_cast<const __nv_bfloat162*>(&w);
  }
  static __device__ __forceinline__ float value(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
  using Bits = uint16_t;
  static __device__ __forceinline__ __nv_bfloat16 make(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Elem<__half> {
  static constexpr int N = 8;
  static constexpr uint32_t kNegInf = 0xFC00FC00u;
  static __device__ __forceinline__ void unpack(uint4 q, float2* x) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
  }
  static __device__ __forceinline__ uint4 pack(const float2* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(x[i].x, x[i].y);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(const __half* p) { return __half2float(*p); }
  using Max = __half2;  // two at a time, without widening
  static __device__ __forceinline__ Max max_of(Max m, uint4 q) {
    const __half2* h = reinterpret_cast<const __half2*>(&q);
    return __hmax2(__hmax2(__hmax2(m, h[0]), __hmax2(h[1], h[2])), h[3]);
  }
  static __device__ __forceinline__ Max none() {
    const uint32_t w = kNegInf;
    return *reinterpret_cast<const __half2*>(&w);
  }
  static __device__ __forceinline__ float value(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
  using Bits = uint16_t;
  static __device__ __forceinline__ __half make(float x) { return __float2half_rn(x); }
};

// The 128 bits of a piece moved by one element towards its end or its start,
// with the element that comes in or has gone out (edges of a row only).
__device__ __forceinline__ void push_front(uint4& q, uint32_t bits, float) {
  q = make_uint4(bits, q.x, q.y, q.z);
}
template <typename T>
__device__ __forceinline__ void push_front(uint4& q, uint32_t bits, T) {
  q.w = __funnelshift_l(q.z, q.w, 16);
  q.z = __funnelshift_l(q.y, q.z, 16);
  q.y = __funnelshift_l(q.x, q.y, 16);
  q.x = (q.x << 16) | bits;
}
__device__ __forceinline__ uint32_t pop_front(uint4& q, float) {
  const uint32_t bits = q.x;
  q = make_uint4(q.y, q.z, q.w, 0u);
  return bits;
}
template <typename T>
__device__ __forceinline__ uint32_t pop_front(uint4& q, T) {
  const uint32_t bits = q.x & 0xFFFFu;
  q.x = __funnelshift_r(q.x, q.y, 16);
  q.y = __funnelshift_r(q.y, q.z, 16);
  q.z = __funnelshift_r(q.z, q.w, 16);
  q.w >>= 16;
  return bits;
}

}  // namespace meq

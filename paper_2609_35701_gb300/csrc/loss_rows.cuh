// Rows of logits in registers: their pieces, statistics and gradients, shared
// by the kernels of the losses.
#pragma once

#include <cfloat>
#include <cmath>

#include "meq_elem.cuh"
#include "meq_elementwise.cuh"

namespace meq {
namespace loss {

constexpr float kLog2e = 1.4426950216293335f;  // and kLog2eLo

struct RowArgs {
  const void* logits;
  int64_t rows, cols, ld;
  const int64_t* targets;
  const float* old_logp;
  const float* advantages;
  const float* weights;     // NULL: 1
  const float* ref_logp;
  float clip_lo, clip_hi, kl;
  const float* grad_scale;  // NULL: 1
  float* logp;              // out
  float* lse;               // out, may be NULL
  float2* stat;             // statistics pass: max and sum of exponentials, may be NULL
  float* coef;              // statistics pass: zeroed, may be NULL
  float4* terms;            // policy: per row, weighted {loss, surrogate, k3, clipped}
  void* grad;               // NULL: none
  int64_t ld_grad;
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The largest of the warp's values, NaN aside.
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// exp(a - b) for the few joins of statistics (0 for a = -inf and any finite b)
__device__ __forceinline__ float exp_diff(float a, float b) { return exp2_approx((a - b) * kLog2e); }

// exp(x - m) as 2^(x log2e - c) with c = m log2e rounded: one multiply-add per
// element (its product is not rounded, so no x overflows it), and the rounding
// of c undone once, by the factor `fix`. m: finite, at most kFar in magnitude,
// where c is off by less than 0.1. log2e in two parts: the first alone is off
// by 1.3e-8 of itself, which would bias a sum by as much per unit of m - x; a
// single element can do without the second part (fix_hi).
constexpr float kLog2eLo = 1.9259629911266175e-8f;
constexpr float kFar = 1e6f;
struct ExpBase {
  float c, fix, fix_hi;
  __device__ __forceinline__ explicit ExpBase(float m) {
    c = m * kLog2e;
    const float off = fmaf(m, kLog2e, -c);
    fix = exp2_approx(-fmaf(m, kLog2eLo, off));
    fix_hi = exp2_approx(-off);
  }
};
// The exponential of one element relative to c, as the sums take it.
__device__ __forceinline__ float exp_at(float x, float c) { return exp2_approx(fmaf(x, kLog2eLo, fmaf(x, kLog2e, -c))); }

// A row cut at the 16-byte boundaries of its address: piece k holds elements
// k N - lead .. k N - lead + N - 1 of the row, as far as they exist. Pieces
// `begin` .. `end` - 1 exist whole; at most the first and the last do not. A
// warp takes chunks of 32 P consecutive pieces, lane l pieces l, l + 32, .. of
// it: of a chunk that exists whole every access has a fixed distance from the
// lane's first, and only the row's first and last chunk look at their pieces
// one by one.
template <typename T>
struct Row {
  static constexpr int N = Elem<T>::N;
  using Bits = typename Elem<T>::Bits;
  const T* p;  // element 0
  int cols;
  int lead;    // elements of the first 16 bytes that precede the row
  int pieces, begin, end;
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t ld, int64_t cols_)
      : p(static_cast<const T*>(base) + row * ld), cols(static_cast<int>(cols_)) {
    lead = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    pieces = (cols + lead + N - 1) / N;
    begin = lead > 0 ? 1 : 0;
    end = (cols + lead) / N;
  }
  // A piece that does not exist whole, element by element.
  __device__ __forceinline__ uint4 load_part(int k) const {
    const Bits* b = reinterpret_cast<const Bits*>(p);
    uint4 q = none();
#pragma unroll
    for (int e = N - 1; e >= 0; --e) {
      const int i = k * N - lead + e;
      push_front(q, i >= 0 && i < cols ? b[i] : static_cast<Bits>(Elem<T>::kNegInf), T());
    }
    return q;
  }
  __device__ __forceinline__ void store_part(T* g, int k, uint4 q) const {
    Bits* b = reinterpret_cast<Bits*>(g);
#pragma unroll 1
    for (int i = k * N - lead; i < k * N - lead + N; ++i) {
      const uint32_t bits = pop_front(q, T());
      if (i >= 0 && i < cols) b[i] = static_cast<Bits>(bits);
    }
  }
  static __device__ __forceinline__ uint4 none() {
    return make_uint4(Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf);
  }
  // Whether the row's last piece is a part, and this lane's (as its piece last_of / 32).
  template <int P>
  __device__ __forceinline__ bool last_part(int k0, int* last_of) const {
    *last_of = pieces - 1 - k0;
    return pieces > end && pieces > begin && *last_of >= 0 && *last_of < 32 * P && *last_of % 32 == 0;
  }
  // Pieces k0 + 32 j of the chunk that starts at piece `first` (-inf where there is none); k0 = first + lane.
  template <int P>
  __device__ __forceinline__ void load(int first, int k0, uint4 (&q)[P]) const {
    const uint4* s = reinterpret_cast<const uint4*>(p + (k0 * N - lead));
    if (first >= begin && first + 32 * P <= end) {
#pragma unroll
      for (int j = 0; j < P; ++j) q[j] = __ldcs(s + 32 * j);
      return;
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int k = k0 + 32 * j;
      q[j] = none();
      if (k >= begin && k < end) q[j] = __ldcs(s + 32 * j);
    }
    if (k0 < begin) q[0] = load_part(0);
    int last;
    if (last_part<P>(k0, &last)) {
      const uint4 x = load_part(pieces - 1);
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (32 * j == last) q[j] = x;
    }
  }
  // f(x) of each piece x = q[j] into the gradient's row g. `same`: g has the same offset in its 16 bytes as p.
  template <int P, typename F>
  __device__ __forceinline__ void store(T* g, bool same, int first, int k0, const uint4 (&q)[P], F f) const {
    uint4* d = reinterpret_cast<uint4*>(g + (k0 * N - lead));
    if (same && first >= begin && first + 32 * P <= end) {
#pragma unroll
      for (int j = 0; j < P; ++j) __stcs(d + 32 * j, f(q[j]));
    } else if (same) {
      int last;
      const bool part = last_part<P>(k0, &last);
      uint4 x = q[0];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const int k = k0 + 32 * j;
        if (k >= begin && k < end) __stcs(d + 32 * j, f(q[j]));
        if (32 * j == last) x = q[j];
      }
      if (k0 < begin) store_part(g, 0, f(q[0]));
      if (part) store_part(g, pieces - 1, f(x));
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (k0 + 32 * j < pieces) store_part(g, k0 + 32 * j, f(q[j]));
    }
  }
};

__device__ __forceinline__ bool same_offset(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// What turns logits into gradients: c ([j = target] - exp(z_j - top) / sum).
struct GradScale {
  float c, base, neg;  // neg = -c / sum with the base's fix
  bool far;            // |top| above kFar (masks of a type's lowest value, all of a row's): exp(z - top) step by step
  float top;
  GradScale() = default;
  __device__ __forceinline__ GradScale(float c_, float top_, float sum) : c(c_), top(top_) {
    far = !(fabsf(top_) <= kFar);
    const ExpBase b(far ? 0.f : top_);
    base = b.c;
    neg = -c_ / sum * b.fix_hi;
  }
  // of tokens that are not the target
  template <bool kFarTop>
  __device__ __forceinline__ float2 other(float2 x) const {
    if (kFarTop) return make_float2(exp_diff(x.x, top) * neg, exp_diff(x.y, top) * neg);
    x = fma2(x, make_float2(kLog2e, kLog2e), make_float2(-base, -base));
    return mul2(make_float2(exp2_approx(x.x), exp2_approx(x.y)), make_float2(neg, neg));
  }
  template <bool kFarTop, typename T>
  __device__ __forceinline__ uint4 piece(uint4 q) const {
    float2 x[Elem<T>::N / 2];
    Elem<T>::unpack(q, x);
#pragma unroll
    for (int e = 0; e < Elem<T>::N / 2; ++e) x[e] = other<kFarTop>(x[e]);
    return Elem<T>::pack(x);
  }
  __device__ __forceinline__ float at_target(float zt) const {
    const float2 x = make_float2(zt, zt);
    return (far ? other<true>(x) : other<false>(x)).x + c;
  }
};
// Whether this lane holds the target's piece (no lane does for kNoToken).
constexpr int kNoToken = -(1 << 30);
template <typename T, int P>
__device__ __forceinline__ bool holds(const Row<T>& r, int k0, int target) {
  const unsigned at = static_cast<unsigned>((target + r.lead) / Elem<T>::N - k0);
  return at < 32u * P && at % 32u == 0u;
}
// The gradient of a chunk. The target's token is written once more, by the
// thread that has just written its piece (and alone needs zt).
template <bool kFarTop, typename T, int P>
__device__ __forceinline__ void store_grad_of(const Row<T>& r, T* g, bool same, int first, int k0, const uint4 (&q)[P],
                                              const GradScale& s) {
  r.template store<P>(g, same, first, k0, q, [&](uint4 piece) { return s.template piece<kFarTop, T>(piece); });
}
template <typename T, int P>
__device__ __forceinline__ void store_grad(const Row<T>& r, T* g, bool same, int first, int k0, const uint4 (&q)[P],
                                           const GradScale& s, int target, float zt) {
  if (s.far) store_grad_of<true>(r, g, same, first, k0, q, s);
  else store_grad_of<false>(r, g, same, first, k0, q, s);
  if (holds<T, P>(r, k0, target)) g[target] = Elem<T>::make(s.at_target(zt));
}
template <typename T, int P>
__device__ __forceinline__ void store_zeros(const Row<T>& r, T* g, bool same, int first, int k0) {
  const uint4 q[P] = {};
  r.template store<P>(g, same, first, k0, q, [](uint4 piece) { return piece; });
}

// Maximum and sum of exponentials relative to it. The maximum's own is exactly 1
// in the sum (the approximate one is taken off again, and the rest made
// relative to the maximum), so that a token of probability one has the
// log-probability 0.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  MaxSum r;
  r.m = fmaxf(a.m, b.m);
  const float base = finite_or_zero(r.m);
  r.s = a.s * exp_diff(a.m, base) + b.s * exp_diff(b.m, base);
  return r;
}

// z - log(sum_j exp(z_j)) from a row's maximum m and sum s, rounded about once:
// z - m and the part of log(s) that its exponent gives, a multiple of log(2),
// are added with their rounding errors, and log of s's significand, below
// log(2), joins those. (The log-ratios of an answer are summed over hundreds of
// tokens: half an ulp of lse and of log(s) each, and any common bias, show.)
constexpr float kLn2 = 0.693147182f, kLn2Lo = -1.90465421e-9f;  // log(2) in two parts
// ex2.approx is low by 5.0e-8 of its value on average for negative arguments (measured over [-20, 0]): the sum is,
// but for the maximum's own 1.
constexpr float kExpBias = 5.0e-8f;
__device__ __forceinline__ float two_sum(float a, float b, float* error) {
  const float s = __fadd_rn(a, b), v = __fadd_rn(s, -a);
  *error = __fadd_rn(__fadd_rn(a, -__fadd_rn(s, -v)), __fadd_rn(b, -v));
  return s;
}
// *rest: what the last rounding took off.
__device__ __forceinline__ float log_prob(float z, MaxSum t, float* rest) {
  *rest = 0.f;
  if (!(t.s >= FLT_MIN && t.s <= FLT_MAX)) return (z - t.m) - logf(t.s);
  const uint32_t bits = __float_as_uint(t.s);
  const float k = static_cast<float>(static_cast<int>(bits >> 23) - 127);
  const float log_part = logf(__uint_as_float((bits & 0x007FFFFFu) | 0x3F800000u));
  const float ln = __fmul_rn(k, kLn2), off = fmaf(k, kLn2, -ln);
  float e0, e1;
  const float d = two_sum(z, -t.m, &e0), r = two_sum(d, -ln, &e1);
  const float bias = __fdividef(kExpBias * (t.s - 1.f), t.s);
  const float tail = (e0 + e1) - ((off + fmaf(k, kLn2Lo, bias)) + log_part);
  if (!(fabsf(d) <= FLT_MAX)) return d;  // an infinite d has no error terms
  return two_sum(r, tail, rest);
}
__device__ __forceinline__ float log_prob(float z, MaxSum t) {
  float rest;
  return log_prob(z, t, &rest);
}

// The policy loss of one token: its terms, unweighted, and dL/dlogp. The ratio is
// of logp + rest: half an ulp of a log-probability, 5e-7 at -11, is most of the
// error of a sum of advantages that cancel.
struct TokenLoss {
  float surrogate, k3, clipped, slope;
};
__device__ __forceinline__ TokenLoss policy_token(float logp, float rest, float old_logp, float adv, const float* ref, float lo, float hi,
                                                  float kl) {
  TokenLoss t;
  const float ratio = expf((logp - old_logp) + rest);
  const float plain = ratio * adv, bounded = fminf(fmaxf(ratio, lo), hi) * adv;
  const bool cut = plain > bounded;
  // a NaN ratio stays one: neither comparison holds for it
  t.surrogate = cut ? -bounded : -plain;
  t.slope = cut ? 0.f : -plain;
  t.clipped = cut ? 1.f : 0.f;
  t.k3 = 0.f;
  if (kl != 0.f) {
    const float d = (*ref - logp) - rest;
    const float em = expm1f(d);
    t.k3 = em - d;
    t.slope -= kl * em;
  }
  return t;
}

// Statistics in one pass (kPolicy 0) or the policy loss and its gradient, rows
// streamed through shared memory. False: the rows do not suit it.
bool stream_suits(int64_t rows, int64_t cols, int elem_bytes, bool policy);
cudaError_t launch_stream(const RowArgs& a, int type, bool policy, cudaStream_t st);
// The limit of the streamed kernel's waits (0: the usual one) and a row whose data never comes (-1: none), for the
// calling thread's next launches.
void stream_wait(unsigned long long ns, int64_t withheld);

}  // namespace loss
}  // namespace meq

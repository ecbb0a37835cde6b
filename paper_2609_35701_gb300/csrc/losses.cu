// Losses of fine-tuning on token log-probabilities, and the gradient of the
// logits: token log-probabilities, the clipped policy loss with its KL term,
// and the paired preference loss.
//
// For a row of logits z with target t:  lse = log sum_j exp(z_j),
// logp = z_t - lse,  d logp / d z_j = [j = t] - exp(z_j - lse). Every loss here
// is a function of the rows' logp, so the gradient of a row is one coefficient
// c = dL/dlogp times ([j = t] - softmax_j).
//
// Policy loss: c depends on the row alone. A row is read once, held in
// registers (8 pieces of 16 bytes per thread) by one CTA or a cluster of up to
// 8, reduced (warp, CTA, then the cluster's CTAs through distributed shared
// memory) and its gradient written from the registers: the traffic is one read
// and one write of the logits, the floor. Rows that no cluster holds take
// three launches (statistics, coefficients, gradient).
//
// Preference loss: c needs the sums over the two answers of a pair, so the
// logits are read again for the gradient, last rows first: those are the ones
// that the statistics pass left in L2.
//
// Rows start at any element: a row is cut at the 16-byte boundaries of its
// address, and only its first and last piece are moved element by element.
// Sums and statistics are fp32 or wider; exponentials are of z - max.
#include <cfloat>
#include <cmath>
#include <new>
#include <string>

#include "../../include/meq.h"
#include "meq_elementwise.cuh"

using namespace meq;

namespace {

constexpr int kPieces = 8;          // 16-byte pieces per thread
constexpr int kChunkPieces = 32 * kPieces;  // of a warp
constexpr int kMaxCluster = 8;
constexpr int kRowThreads = 512;    // most threads of a CTA before the cluster grows
constexpr int kRowThreadsMax = 1024;
constexpr int kGradThreads = 256;
constexpr int kGradPieces = 4;
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
// Two fp32 operations in one instruction, each rounded as a single one is.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(d)
      : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)), "l"(*reinterpret_cast<uint64_t*>(&c)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&d);
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

template <typename T>
struct Elem;  // 16-bit and 32-bit logits
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
                                              const GradScale& s, int target, float zt) {
  constexpr int H = Elem<T>::N / 2;
  r.template store<P>(g, same, first, k0, q, [&](uint4 piece) {
    float2 x[H];
    Elem<T>::unpack(piece, x);
#pragma unroll
    for (int e = 0; e < H; ++e) x[e] = s.template other<kFarTop>(x[e]);
    return Elem<T>::pack(x);
  });
  if (holds<T, P>(r, k0, target)) g[target] = Elem<T>::make(s.template other<kFarTop>(make_float2(zt, zt)).x + s.c);
}
template <typename T, int P>
__device__ __forceinline__ void store_grad(const Row<T>& r, T* g, bool same, int first, int k0, const uint4 (&q)[P],
                                           const GradScale& s, int target, float zt) {
  if (s.far) store_grad_of<true>(r, g, same, first, k0, q, s, target, zt);
  else store_grad_of<false>(r, g, same, first, k0, q, s, target, zt);
}
template <typename T, int P>
__device__ __forceinline__ void store_zeros(const Row<T>& r, T* g, bool same, int first, int k0) {
  const uint4 q[P] = {};
  r.template store<P>(g, same, first, k0, q, [](uint4 piece) { return piece; });
}

// Running maximum and sum of exponentials relative to it.
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

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}

struct RowShared {
  MaxSum warp[32];
  MaxSum cta[kMaxCluster];
};

// The maximum and sum of the whole row from each warp's, for every thread of
// the cluster, in an order that does not depend on timing.
__device__ __forceinline__ MaxSum row_join(MaxSum w, RowShared& sh, uint32_t rank, uint32_t ctas) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) sh.warp[threadIdx.x >> 5] = w;
  __syncthreads();
  MaxSum t{-INFINITY, 0.f};
  if (lane < warps) t = sh.warp[lane];
  float m = t.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  t.s *= exp_diff(t.m, finite_or_zero(m));
  t.m = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t.s += __shfl_xor_sync(0xffffffffu, t.s, o);
  if (ctas == 1) return t;
  // every CTA of the cluster has begun (the wait of the arrive at the kernel's start)
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (threadIdx.x < ctas) {
    const uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(&sh.cta[rank]));
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(remote), "f"(t.m), "f"(t.s) : "memory");
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  MaxSum r = sh.cta[0];
  for (uint32_t i = 1; i < ctas; ++i) r = join(r, sh.cta[i]);
  return r;
}

// max and sum of exponentials over a warp's pieces, for all its lanes
template <typename T>
__device__ __forceinline__ MaxSum warp_stats(const uint4 (&q)[kPieces]) {
  MaxSum w;
  typename Elem<T>::Max top = Elem<T>::none();
#pragma unroll
  for (int j = 0; j < kPieces; ++j) top = Elem<T>::max_of(top, q[j]);
  float m = Elem<T>::value(top);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  w.m = m;
  constexpr int H = Elem<T>::N / 2;
  float2 s = make_float2(0.f, 0.f);
  if (fabsf(m) <= kFar || m == -INFINITY) {
    const ExpBase b(finite_or_zero(m));
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      float2 x[H];
      Elem<T>::unpack(q[j], x);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const float2 y = fma2(x[e], make_float2(kLog2e, kLog2e), make_float2(-b.c, -b.c));
        const float2 z = fma2(x[e], make_float2(kLog2eLo, kLog2eLo), y);
        s = add2(s, make_float2(exp2_approx(z.x), exp2_approx(z.y)));
      }
    }
    w.s = (s.x + s.y) * b.fix;
  } else {
    // far from zero (+inf gives NaN)
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      float2 x[H];
      Elem<T>::unpack(q[j], x);
#pragma unroll
      for (int e = 0; e < H; ++e) s = add2(s, make_float2(exp_diff(x[e].x, m), exp_diff(x[e].y, m)));
    }
    w.s = s.x + s.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) w.s += __shfl_xor_sync(0xffffffffu, w.s, o);
  return w;
}

// The policy loss of one token: its terms, unweighted, and dL/dlogp.
struct TokenLoss {
  float surrogate, k3, clipped, slope;
};
__device__ __forceinline__ TokenLoss policy_token(float logp, float old_logp, float adv, const float* ref, float lo, float hi,
                                                  float kl) {
  TokenLoss t;
  const float ratio = expf(logp - old_logp);
  const float plain = ratio * adv, bounded = fminf(fmaxf(ratio, lo), hi) * adv;
  const bool cut = plain > bounded;
  // a NaN ratio stays one: neither comparison holds for it
  t.surrogate = cut ? -bounded : -plain;
  t.slope = cut ? 0.f : -plain;
  t.clipped = cut ? 1.f : 0.f;
  t.k3 = 0.f;
  if (kl != 0.f) {
    const float d = *ref - logp;
    const float em = expm1f(d);
    t.k3 = em - d;
    t.slope -= kl * em;
  }
  return t;
}

// One CTA or cluster per row. kPolicy: the whole row is in registers, and its
// loss and gradient follow; else the row's statistics alone, in as many rounds
// as it takes.
template <typename T, bool kPolicy>
__global__ void __launch_bounds__(kRowThreadsMax) row_kernel(const RowArgs a) {
  pdl_allow_dependents();
  __shared__ RowShared sh;
  const uint32_t ctas = cluster_size(), rank = ctas == 1 ? 0u : cluster_rank();
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  pdl_wait_predecessor();
  const int64_t row = blockIdx.x / ctas;
  const Row<T> r(a.logits, row, a.ld, a.cols);
  const int64_t target = a.targets[row];
  float w = 1.f;
  if (a.weights) w = a.weights[row];
  const int warps = static_cast<int>(blockDim.x >> 5);
  const int first = (static_cast<int>(rank) * warps + static_cast<int>(threadIdx.x >> 5)) * kChunkPieces;  // the warp's chunk
  const int k0 = first + static_cast<int>(threadIdx.x & 31);
  T* g = nullptr;
  if (kPolicy && a.grad) g = static_cast<T*>(a.grad) + row * a.ld_grad;
  const bool same = same_offset(r.p, g);
  const bool leader = rank == 0 && threadIdx.x == 0;
  if (target < 0 || w == 0.f) {  // not scored: the logits are not read
    if (leader) {
      a.logp[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
      if (a.stat) a.stat[row] = make_float2(0.f, 1.f);
      if (a.coef) a.coef[row] = 0.f;
      if (kPolicy) a.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (kPolicy && g) store_zeros<T, kPieces>(r, g, same, first, k0);
    if (ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    return;
  }
  // beyond the row: no such token, everything that depends on it is NaN
  const int token = target < a.cols ? static_cast<int>(target) : kNoToken;
  const float zt = token != kNoToken ? Elem<T>::get(r.p + token) : __int_as_float(0x7fc00000);
  uint4 q[kPieces];
  MaxSum ws{-INFINITY, 0.f};
  if (kPolicy) {
    r.load(first, k0, q);
    ws = warp_stats<T>(q);
  } else {
    const int step = static_cast<int>(ctas) * warps * kChunkPieces;
    for (int k = 0; first + k < r.pieces; k += step) {
      r.load(first + k, k0 + k, q);
      ws = join(ws, warp_stats<T>(q));
    }
  }
  const MaxSum all = row_join(ws, sh, rank, ctas);
  const float logs = logf(all.s);
  const float logp = (zt - all.m) - logs;
  if (!kPolicy) {
    if (leader) {
      a.logp[row] = logp;
      if (a.lse) a.lse[row] = all.m + logs;
      if (a.stat) a.stat[row] = make_float2(all.m, all.s);
      if (a.coef) a.coef[row] = 0.f;
    }
    return;
  }
  const TokenLoss t = policy_token(logp, a.old_logp[row], a.advantages[row], a.ref_logp + row, a.clip_lo, a.clip_hi, a.kl);
  if (leader) {
    a.logp[row] = logp;
    a.terms[row] = make_float4(w * (t.surrogate + a.kl * t.k3), w * t.surrogate, w * t.k3, w * t.clipped);
  }
  if (!g) return;
  const float c = w * t.slope * (a.grad_scale ? *a.grad_scale : 1.f);
  if (c == 0.f) {
    store_zeros<T, kPieces>(r, g, same, first, k0);
    return;
  }
  store_grad(r, g, same, first, k0, q, GradScale(c, all.m, all.s), token, zt);
}

// The policy terms and coefficients of rows whose statistics are known.
__global__ void __launch_bounds__(kThreads) policy_terms_kernel(const RowArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (row >= a.rows) return;
  const float w = a.weights ? a.weights[row] : 1.f;
  float4 terms = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.targets[row] >= 0 && w != 0.f) {
    const TokenLoss t = policy_token(a.logp[row], a.old_logp[row], a.advantages[row], a.ref_logp + row, a.clip_lo, a.clip_hi, a.kl);
    terms = make_float4(w * (t.surrogate + a.kl * t.k3), w * t.surrogate, w * t.k3, w * t.clipped);
    a.coef[row] = w * t.slope * (a.grad_scale ? *a.grad_scale : 1.f);
  }
  a.terms[row] = terms;
}

// Gradient of the logits from each row's statistics and coefficient, the last rows first.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) grad_kernel(const RowArgs a, int tiles, int64_t blocks) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int64_t row = a.rows - 1 - b / tiles;
    const Row<T> r(a.logits, row, a.ld, a.cols);
    const int first = (static_cast<int>(b % tiles) * (kGradThreads / 32) + static_cast<int>(threadIdx.x >> 5)) * 32 * kGradPieces;
    const int k0 = first + static_cast<int>(threadIdx.x & 31);
    T* g = static_cast<T*>(a.grad) + row * a.ld_grad;
    const bool same = same_offset(r.p, g);
    const float c = a.coef[row];
    if (c == 0.f) {
      store_zeros<T, kGradPieces>(r, g, same, first, k0);
      continue;
    }
    const float2 stat = a.stat[row];
    const int64_t target = a.targets[row];
    uint4 q[kGradPieces];
    r.load(first, k0, q);
    const int token = target < a.cols ? static_cast<int>(target) : kNoToken;
    // read by the thread that will write it, since the gradient may lie in the logits' place
    const float zt = holds<T, kGradPieces>(r, k0, token) ? Elem<T>::get(r.p + token) : 0.f;
    store_grad(r, g, same, first, k0, q, GradScale(c, stat.x, stat.y), token, zt);
  }
}

// One block per pair: the weighted sums of logp - ref over the two answers,
// the loss, and the coefficients of their rows.
__global__ void __launch_bounds__(kThreads) pair_kernel(const RowArgs a, const int64_t* __restrict__ starts, float beta,
                                                        float smoothing, float inv_pairs, float* __restrict__ margins,
                                                        float* __restrict__ pair_loss) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[kThreads / 32];
  const int64_t j = blockIdx.x;
  const int64_t s0 = starts[2 * j], s1 = starts[2 * j + 1], s2 = starts[2 * j + 2];
  if (!(0 <= s0 && s0 <= s1 && s1 <= s2 && s2 <= a.rows)) {  // no such answers: NaN, and no gradient
    if (threadIdx.x == 0) margins[j] = pair_loss[j] = __int_as_float(0x7fc00000);
    return;
  }
  WideSum d;
  for (int64_t i = s0 + threadIdx.x; i < s2; i += kThreads) {
    const float w = a.weights ? a.weights[i] : 1.f;
    if (a.targets[i] < 0 || w == 0.f) continue;
    const float x = w * (a.logp[i] - a.ref_logp[i]);
    d.add(i < s1 ? x : -x);
  }
  const float x = beta * block_total(d, sh);
  // -log sigma(y) = max(-y, 0) + log(1 + exp(-|y|))
  const float e = expf(-fabsf(x)), tail = log1pf(e);
  const float sigma = x >= 0.f ? 1.f / (1.f + e) : e / (1.f + e);
  // sigma(-x) = 1 - sigma(x) without its cancellation
  const float anti = x >= 0.f ? e / (1.f + e) : 1.f / (1.f + e);
  if (threadIdx.x == 0) {
    margins[j] = x;
    pair_loss[j] = inv_pairs * ((1.f - smoothing) * (fmaxf(-x, 0.f) + tail) + smoothing * (fmaxf(x, 0.f) + tail));
  }
  if (!a.grad) return;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float slope = (smoothing * sigma - (1.f - smoothing) * anti) * beta * inv_pairs * gs;
  for (int64_t i = s0 + threadIdx.x; i < s2; i += kThreads) {
    const float w = a.weights ? a.weights[i] : 1.f;
    if (a.targets[i] < 0 || w == 0.f) continue;
    a.coef[i] = w * (i < s1 ? slope : -slope);
  }
}

// sums[k] = sum of terms[i * K + k] over n rows, in a fixed order.
constexpr int kSumThreads = 512;
template <int K>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const float* __restrict__ terms, int64_t n, float* __restrict__ sums) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[K][kSumThreads / 32];
  WideSum s[K];
  for (int64_t i = threadIdx.x; i < n; i += kSumThreads) {
    float x[K];
    if (K == 4) {
      const float4 q = reinterpret_cast<const float4*>(terms)[i];
      x[0] = q.x, x[1 % K] = q.y, x[2 % K] = q.z, x[3 % K] = q.w;
    } else {
      x[0] = terms[i];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) s[k].add(x[k]);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const float t = block_total(s[k], sh[k]);
    if (threadIdx.x == 0) sums[k] = t;
  }
}

// ------------------------------------------------------------------- host
meq_status fail(meq_status s, const std::string& msg) {
  meq::set_global_error(msg);
  return s;
}
meq_status launch_status(cudaError_t e, const char* fn, const char* what) {
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

int elem_bytes(int type) { return type == MEQ_F32 ? 4 : 2; }

// How a row of `cols` elements is spread over a cluster.
struct RowShape {
  int ctas, threads;
  bool held;  // the row fits into the cluster's registers
};
RowShape row_shape(int64_t rows, int64_t cols, int type, int sms) {
  const int n = 16 / elem_bytes(type);
  const int64_t pieces = (cols + 2 * n - 2) / n;  // of a row that starts anywhere
  RowShape s{1, 32, true};
  auto need = [&](int ctas) { return (pieces + static_cast<int64_t>(ctas) * kPieces - 1) / (static_cast<int64_t>(ctas) * kPieces); };
  while (s.ctas < kMaxCluster && need(s.ctas) > kRowThreads) s.ctas *= 2;
  // few rows: more SMs to each
  while (s.ctas < kMaxCluster && rows * s.ctas * 2 <= 2 * sms && need(s.ctas) > 64) s.ctas *= 2;
  const int64_t t = (need(s.ctas) + 31) / 32 * 32;
  s.held = t <= kRowThreadsMax;
  s.threads = static_cast<int>(s.held ? t : kRowThreads);
  return s;
}

template <bool kPolicy>
cudaError_t launch_rows_of(const RowArgs& a, int type, const RowShape& s, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.rows * s.ctas)), block(s.threads);
  if (type == MEQ_F32) return launch_pdl(row_kernel<float, kPolicy>, grid, block, 0, st, s.ctas, a);
  if (type == MEQ_BF16) return launch_pdl(row_kernel<__nv_bfloat16, kPolicy>, grid, block, 0, st, s.ctas, a);
  return launch_pdl(row_kernel<__half, kPolicy>, grid, block, 0, st, s.ctas, a);
}

cudaError_t launch_grad(const RowArgs& a, int type, cudaStream_t st) {
  const int n = 16 / elem_bytes(type);
  const int64_t pieces = (a.cols + 2 * n - 2) / n, per = kGradPieces * kGradThreads;
  const int tiles = static_cast<int>((pieces + per - 1) / per);
  const int64_t blocks = a.rows * tiles;
  const dim3 grid(static_cast<unsigned>(blocks < 0x40000000 ? blocks : 0x40000000)), block(kGradThreads);
  if (type == MEQ_F32) return launch_pdl(grad_kernel<float>, grid, block, 0, st, 1, a, tiles, blocks);
  if (type == MEQ_BF16) return launch_pdl(grad_kernel<__nv_bfloat16>, grid, block, 0, st, 1, a, tiles, blocks);
  return launch_pdl(grad_kernel<__half>, grid, block, 0, st, 1, a, tiles, blocks);
}

int device_sms(cudaError_t* e) {
  int dev = 0, sms = 0;
  *e = cudaGetDevice(&dev);
  if (*e == cudaSuccess) *e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// The checks that the three calls share; an empty text: fine.
std::string check_logits(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                         const float* logp) {
  if (type != MEQ_F32 && type != MEQ_BF16 && type != MEQ_F16) return "type must be a meq_dtype";
  if (rows < 0 || rows > (int64_t(1) << 27)) return "rows must be in 0..2^27";
  if (cols < 1 || cols > (int64_t(1) << 28)) return "cols must be in 1..2^28";
  if (rows > 1 && ld < cols) return "the row stride must be at least cols";
  if (ld < 0 || ld > (int64_t(1) << 40)) return "the row stride must be in 0..2^40";
  if (rows > 0 && (!logits || !targets || !logp)) return "logits, targets and logp must not be NULL";
  if (!aligned_to(logits, elem_bytes(type)) || !aligned_to(targets, 8) || !aligned_to(logp, 4))
    return "a pointer is not aligned to its type";
  return "";
}
std::string check_grad(const void* grad, int64_t ld_grad, int type, int64_t rows, int64_t cols, const float* grad_scale,
                       const float* work) {
  if (!work || !aligned_to(work, 16)) return "work must not be NULL and be 16-byte aligned";
  if (grad && rows > 1 && ld_grad < cols) return "the gradient's row stride must be at least cols";
  if (grad && (ld_grad < 0 || ld_grad > (int64_t(1) << 40))) return "the gradient's row stride must be in 0..2^40";
  if (!aligned_to(grad, elem_bytes(type)) || !aligned_to(grad_scale, 4)) return "a pointer is not aligned to its type";
  return "";
}

}  // namespace

extern "C" {

meq_status meq_token_logprobs(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                              float* logp, float* lse, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    const std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_token_logprobs: " + why);
    if (!aligned_to(lse, 4)) return fail(MEQ_ERR_INVALID_ARG, "meq_token_logprobs: a pointer is not aligned to its type");
    if (rows == 0) return MEQ_OK;
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_token_logprobs", "device attributes");
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets, a.logp = logp, a.lse = lse;
    return launch_status(launch_rows_of<false>(a, type, row_shape(rows, cols, type, sms), static_cast<cudaStream_t>(cuda_stream)),
                         "meq_token_logprobs", "launch");
  });
}

int64_t meq_loss_work_floats(int64_t rows, int64_t pairs) { return rows < 0 || pairs < 0 ? 0 : 7 * rows + pairs + 4; }

meq_status meq_policy_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                           const float* old_logp, const float* advantages, const float* weights, const float* ref_logp,
                           float clip_low, float clip_high, float kl_coef, float* sums, float* logp, void* grad,
                           int64_t ld_grad, const float* grad_scale, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (why.empty()) why = check_grad(grad, ld_grad, type, rows, cols, grad_scale, work);
    if (why.empty() && rows > 0 && (!old_logp || !advantages)) why = "old_logp and advantages must not be NULL";
    if (why.empty() && (!sums || !aligned_to(sums, 4))) why = "sums must not be NULL";
    if (why.empty() && !(clip_low >= 0.f && clip_low <= 1.f && clip_high >= 0.f && std::isfinite(clip_high)))
      why = "clip_low must be in 0..1 and clip_high finite and >= 0";
    if (why.empty() && !(kl_coef >= 0.f && std::isfinite(kl_coef))) why = "kl_coef must be finite and >= 0";
    if (why.empty() && kl_coef > 0.f && rows > 0 && !ref_logp) why = "a KL term needs ref_logp";
    if (why.empty() && !(aligned_to(old_logp, 4) && aligned_to(advantages, 4) && aligned_to(weights, 4) && aligned_to(ref_logp, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_policy_loss: " + why);
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets;
    a.old_logp = old_logp, a.advantages = advantages, a.weights = weights, a.ref_logp = ref_logp;
    a.clip_lo = 1.f - clip_low, a.clip_hi = 1.f + clip_high, a.kl = kl_coef, a.grad_scale = grad_scale;
    a.logp = logp, a.terms = reinterpret_cast<float4*>(work), a.grad = grad, a.ld_grad = ld_grad;
    if (rows > 0) {
      const RowShape s = row_shape(rows, cols, type, sms);
      if (s.held) {
        e = launch_rows_of<true>(a, type, s, st);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "launch");
      } else {
        a.stat = reinterpret_cast<float2*>(work + 4 * rows), a.coef = work + 6 * rows;
        e = launch_rows_of<false>(a, type, s, st);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "statistics launch");
        e = launch_pdl(policy_terms_kernel, dim3(static_cast<unsigned>((rows + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, 1, a);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "terms launch");
        if (grad) {
          e = launch_grad(a, type, st);
          if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "gradient launch");
        }
      }
    }
    e = launch_pdl(sum_kernel<4>, dim3(1), dim3(kSumThreads), 0, st, 1, static_cast<const float*>(work), rows, sums);
    return launch_status(e, "meq_policy_loss", "sum launch");
  });
}

meq_status meq_preference_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                               const int64_t* starts, int64_t pairs, const float* ref_logp, const float* weights, float beta,
                               float label_smoothing, float* loss, float* margins, float* logp, void* grad, int64_t ld_grad,
                               const float* grad_scale, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (why.empty()) why = check_grad(grad, ld_grad, type, rows, cols, grad_scale, work);
    if (why.empty() && (pairs < 1 || pairs > (int64_t(1) << 27))) why = "pairs must be in 1..2^27";
    if (why.empty() && (!starts || !loss || !margins || (rows > 0 && !ref_logp))) why = "starts, ref_logp, loss and margins must not be NULL";
    if (why.empty() && !(std::isfinite(beta) && beta > 0.f)) why = "beta must be finite and > 0";
    if (why.empty() && !(label_smoothing >= 0.f && label_smoothing <= 1.f)) why = "label_smoothing must be in 0..1";
    if (why.empty() && !(aligned_to(starts, 8) && aligned_to(ref_logp, 4) && aligned_to(weights, 4) && aligned_to(loss, 4) && aligned_to(margins, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_preference_loss: " + why);
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets, a.weights = weights, a.ref_logp = ref_logp;
    a.grad_scale = grad_scale, a.logp = logp, a.stat = reinterpret_cast<float2*>(work + 4 * rows), a.coef = work + 6 * rows;
    a.grad = grad, a.ld_grad = ld_grad;
    float* pair_loss = work + 7 * rows;
    if (rows > 0) {
      e = launch_rows_of<false>(a, type, row_shape(rows, cols, type, sms), st);
      if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "statistics launch");
    }
    e = launch_pdl(pair_kernel, dim3(static_cast<unsigned>(pairs)), dim3(kThreads), 0, st, 1, a, starts, beta, label_smoothing,
                   static_cast<float>(1.0 / static_cast<double>(pairs)), margins, pair_loss);
    if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "pair launch");
    if (grad && rows > 0) {
      e = launch_grad(a, type, st);
      if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "gradient launch");
    }
    e = launch_pdl(sum_kernel<1>, dim3(1), dim3(kSumThreads), 0, st, 1, static_cast<const float*>(pair_loss), pairs, loss);
    return launch_status(e, "meq_preference_loss", "sum launch");
  });
}

}  // extern "C"

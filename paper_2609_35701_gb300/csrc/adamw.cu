// AdamW over many tensors at once, and the norm of their gradients.
//
// For every element of every entry, at step t (g' = s g with the caller's
// coefficient s):
//
//   m <- b1 m + (1 - b1) g'          v <- b2 v + (1 - b2) g'^2
//   p <- (1 - lr wd d) p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// One pass: 28 bytes per element with everything in fp32 (p, m, v read and
// written, g read), so HBM bounds it. A launch covers up to kMaxEntries
// entries, whose pointers travel in the kernel's arguments (no copy to the
// device before a step), and a block a chunk of one entry, longer ones in larger
// states. A warp takes 256 elements at a time, in fp32 as two groups of 128, so
// that every load and store of a warp is one run of 512 bytes and all loads are
// issued before the first is used.
//
// Measured on 67.1M elements, with the time of the bytes at the measured copy
// rate (6.79 TB/s) in brackets, us: fp32 277 (277), bf16 parameters and gradients
// with fp32 moments 222 (218), 8-bit moments 123 (99), the same with fp32 parameters
// 161 (139); the norm of fp32 gradients 42.0 (39.6), of bf16 ones 24.2 (19.8);
// the values of 8-bit moments 108 (99). Tensors that do not start on 16 bytes
// move an element at a time: 285 to 288 in fp32, 230 to 235 in bf16 with fp32
// moments, 166 to 168 and 198 to 208 in 8 bits. A 32-bit step spills 8 bytes per
// thread at the 64 registers that four blocks per SM leave it, at no cost that shows.
//
// 8-bit states, which instructions bound as much as HBM (some 50 per element, 74%
// of the issue slots): 256 elements, one warp's share, have an fp32 scale each for m
// and for r = sqrt(v), the largest |m| and r of the block, and a code per
// element:
//
//   m = S_m sign(q) (q / 127)^2, |q| <= 127       r = S_r (q / 255)^2, 0 <= q <= 255
//
// A quadratic code spends its steps near zero, where most of a block lies, and
// r is coded instead of v because its range is half as wide (in logarithm) and
// because the update divides by r. Both are rounded to the nearest code; an r
// above zero keeps a code of at least one, since the update would otherwise be
// divided by eps alone. The update itself uses the step's m and r as computed,
// before that rounding. Every operation up to the codes is one IEEE rounding
// (no contraction), so the codes do not depend on how a compiler fuses them.
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "../../include/meq.h"
#include "meq_elementwise.cuh"

using namespace meq;

namespace {

constexpr int kBlock = 256;               // elements per scale and per warp
constexpr int kAdamThreads = 256;
// Thread blocks of a step. With 8-bit states a block is one warp: its warps are
// kept busy by computing, get apart, and would wait for each other's ends.
template <int kBits>
struct Step {
  static constexpr int kWarps = kBits == 8 ? 1 : 8;
  static constexpr int kThreads = 32 * kWarps, kPerSm = kBits == 8 ? 24 : 4;
  static constexpr int kTile = kBlock * kWarps;  // elements that a thread block takes at once: one kBlock per warp
  static constexpr int kMinChunk = kTile, kMaxChunk = kBits == 8 ? 4096 : 16384;  // elements that it takes in turn
};
constexpr int kMaxEntries = 256;          // pointers of one launch: 6 KB of its arguments
constexpr int kNormBlocksPerSm = 6;
constexpr int kNormUnit = 2048;           // most elements of a warp's turn in the norm
constexpr int kSkipped = 0x7fffffff;      // value of AdamShared::nonfinite: a step was skipped

struct AdamEntry {  // host
  int64_t numel;
  int64_t off;     // first element in the state's arrays, a multiple of kBlock
  int64_t chunk0;  // first chunk
  float decay;
};
struct __align__(16) Chunk {
  int64_t first;   // element of its entry that it starts at
  int64_t off;     // the same in the state's arrays
  int32_t left;    // elements of the entry in it
  int32_t entry;
  float decay;
  int32_t pad;
};

// What a step needs of the number of steps before it. A step reads one of two,
// which the turn of a block's chunk names, and one of its blocks writes the
// other for the next step; every block moves its own chunk's turn on. So nothing
// that a step reads is written by another block of it, and no block waits for
// others (a ticket per block with the fences that it needs took 1 us of a small
// step and 2 to 6% of a large one in 8 bits). A step that is skipped on the device
// writes neither and does not count.
struct AdamClock {
  double b1t, b2t;     // b1^t, b2^t of the step
  float inv_bc1;       // 1 / (1 - b1^t)
  float inv_sqrt_bc2;  // 1 / sqrt(1 - b2^t)
  long long steps;     // steps done before it
};
struct AdamShared {
  AdamClock clock[2];
  unsigned int norm_ticket;  // blocks of the norm that are done (0 between its launches)
  int nonfinite;             // 0, 1 + entry with a non-finite moment, or kSkipped
};

__host__ __device__ inline void set_clock(AdamClock* c, double b1t, double b2t, long long steps) {
  // only the differences need double, whose division and root are slow on this GPU
  c->b1t = b1t, c->b2t = b2t, c->steps = steps;
  c->inv_bc1 = 1.f / static_cast<float>(1.0 - b1t);
  c->inv_sqrt_bc2 = 1.f / sqrtf(static_cast<float>(1.0 - b2t));
}

struct AdamArgs {
  const Chunk* chunks_of;  // of the state
  uint32_t* turns;         // of the chunks: which clock is this step's
  AdamShared* shared;
  void* m;              // fp32, or int8 codes
  void* v;              // fp32, or uint8 codes of sqrt(v)
  float* m_scale;       // 8-bit states: one per block
  float* r_scale;
  const float* grad_scale;
  double beta1, beta2;
  float b1, one_minus_b1, b2, one_minus_b2, eps, lr, wd;
  float one;             // 1: see sum2
  int32_t entry0, last;  // first entry of this launch; 1: the step's last launch
  int64_t chunk0;        // first chunk of this launch
  void* params[kMaxEntries];
  const void* grads[kMaxEntries];
  void* copies[kMaxEntries];
};

struct NormArgs {
  const Chunk* chunks_of;  // of the state
  AdamShared* shared;
  float* partials;
  float* out;
  float max_norm;
  int32_t entry0, last, part0, parts;  // first partial of this launch; partials of all launches
  int32_t shift, unit;                 // a warp takes `unit` elements at a time, 1 << shift of them per chunk
  int64_t chunk0, chunks;
  const void* grads[kMaxEntries];
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }
// Two 16-bit elements as fp32, and back.
__device__ __forceinline__ float2 wide(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 wide(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t narrow(float x, float y, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Groups of four elements of a lane, kGap apart, as fp32: in wide accesses where
// they are aligned and all there (kVec), else one by one (those beyond n as
// zero). Two groups that are neighbours go as one access of 16-bit elements.
template <int kGap, bool kVec>
__device__ __forceinline__ void load8(const float* p, int n, float* x) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (kVec) {
      const float4 q = __ldcs(reinterpret_cast<const float4*>(p + kGap * j));
      x[4 * j] = q.x, x[4 * j + 1] = q.y, x[4 * j + 2] = q.z, x[4 * j + 3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * j + i] = kGap * j + i < n ? p[kGap * j + i] : 0.f;
    }
  }
}
template <int kGap, bool kVec, typename T>
__device__ __forceinline__ void load8(const T* p, int n, float* x) {
  if (kVec) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint2 q = __ldcs(reinterpret_cast<const uint2*>(p + kGap * j));
      w[2 * j] = q.x, w[2 * j + 1] = q.y;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = wide(w[i], T());
      x[2 * i] = v.x, x[2 * i + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = kGap * (i / 4) + i % 4;
      x[i] = at < n ? to_f(p[at]) : 0.f;
    }
  }
}
template <int kGap, bool kVec>
__device__ __forceinline__ void store8(float* p, int n, const float* x) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (kVec) {
      __stcs(reinterpret_cast<float4*>(p + kGap * j), make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (kGap * j + i < n) p[kGap * j + i] = x[4 * j + i];
    }
  }
}
template <int kGap, bool kVec, typename T>
__device__ __forceinline__ void store8(T* p, int n, const float* x) {
  if (kVec) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = narrow(x[2 * i], x[2 * i + 1], T());
    if (kGap == 4) {
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
      __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
      __stcs(reinterpret_cast<uint2*>(p + kGap), make_uint2(w[2], w[3]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = kGap * (i / 4) + i % 4;
      if (at < n) from_f(x[i], p + at);
    }
  }
}
// Eight neighbouring elements in shared memory.
__device__ __forceinline__ void near8(const float* p, float* x) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float4 q = reinterpret_cast<const float4*>(p)[j];
    x[4 * j] = q.x, x[4 * j + 1] = q.y, x[4 * j + 2] = q.z, x[4 * j + 3] = q.w;
  }
}
template <typename T>
__device__ __forceinline__ void near8(const T* p, float* x) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = wide(w[i], T());
    x[2 * i] = v.x, x[2 * i + 1] = v.y;
  }
}

// The largest magnitude, or NaN if one is NaN.
__device__ __forceinline__ float max_mag(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float warp_max_mag(float x) {
  float r;
  asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rsqrt_approx(float x) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float2 splat(float x) { return make_float2(x, x); }

// a + b rounded once. An addition of two products would be contracted into a
// multiply-add (which add.rn.f32x2 does not keep the assembler from doing); one
// factor that is only known to the launch does.
__device__ __forceinline__ float2 sum2(float2 a, float2 b, float one) { return fma2(a, splat(one), b); }

// A byte as fp32: put below the exponent of 2^23, which is taken off again.
__device__ __forceinline__ float2 two_bytes(uint32_t w, int i) {
  const float2 x = make_float2(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 + i)),
                               __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7541 + i)));
  return x;
}
// Four codes and a scale: scale (code / most)^2, with the code's sign for m.
__device__ __forceinline__ void decode_m4(uint32_t w, float scale, float2* x) {
  w ^= 0x80808080u;  // code + 128
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 t = mul2(add2(two_bytes(w, 2 * i), splat(-8388608.f - 128.f)), splat(1.0f / 127.0f));
    x[i] = mul2(make_float2(__fmul_rn(t.x, fabsf(t.x)), __fmul_rn(t.y, fabsf(t.y))), splat(scale));
  }
}
__device__ __forceinline__ void decode_r4(uint32_t w, float scale, float2* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 t = mul2(add2(two_bytes(w, 2 * i), splat(-8388608.f)), splat(1.0f / 255.0f));
    x[i] = mul2(mul2(t, t), splat(scale));
  }
}
// A block whose largest magnitude is a denormal is held as zero, codes and
// scale: its reciprocal would overflow.
__device__ __forceinline__ float block_scale(float top) { return top >= FLT_MIN ? top : 0.f; }
// The code of x >= 0 before its rounding, most sqrt(x (1 / scale)), every
// operation rounded once.
__device__ __forceinline__ float code_exact(float x, float scale, float most) {
  const float inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  return __fmul_rn(most, __fsqrt_rn(__fmul_rn(x, inv)));
}
// kRound + y holds rint(y) in its low byte, in two's complement.
constexpr float kRound = 12582912.f;  // 1.5 2^23
// Codes y of four elements, rounded and packed. The codes have been formed with
// approximate roots; *worst is the largest distance from a whole number among
// them, so that the caller can see whether one lies too near a half to trust.
__device__ __forceinline__ uint32_t pack_codes(const float2* y, float* worst) {
  float2 z[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    z[i] = add2(y[i], splat(kRound));
    const float2 off = fma2(add2(z[i], splat(-kRound)), splat(-1.f), y[i]);
    *worst = max_mag(*worst, off.x, off.y);
  }
  const uint32_t lo = __byte_perm(__float_as_uint(z[0].x), __float_as_uint(z[0].y), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(z[1].x), __float_as_uint(z[1].y), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}
// The approximate code of m is sqrt.approx of |m| times 127^2 rcp.approx(scale):
// relative errors of 2^-23 each, the product's halved by the root, and those
// of the exact formula, 4.2e-7 in all or 5.3e-5 of 127. r has a root of its own
// and the scale's: 5.4e-7, or 1.4e-4 of 255.
constexpr float kNearM = 0.5f - 7e-5f, kNearR = 0.5f - 1.8e-4f;

// Below this largest v of a block its roots are exact: the approximate root
// takes v < 2^-126 for zero, which decides no code where v is 1e-12 of the
// largest (a fourth root of 1.1e-3, 0.27 of a code), but would in such a block.
constexpr float kSmallV = 1e-26f;
// The largest root that is taken for zero. The update divides by it times
// 1/sqrt(1 - b2^t), plus eps: where eps does not drown it, every root is exact.
constexpr float kLostRoot = 0x1p-63f;

// The approximate codes of m hold for blocks whose largest |m| lies between
// these: below, 127^2 over it comes near overflow (and is infinite under 4.8e-35);
// above, its approximate reciprocal is taken for zero (from 2^126). Codes of
// other blocks are formed exactly.
constexpr float kLeastM = 0x1p-112f, kMostM = 0x1p125f;

// A warp's lane in an entry of the state: its first element there, and in the
// state's arrays.
template <typename P, typename G>
struct Lane {
  P* p;
  const G* g;
  __nv_bfloat16* copy;
  int64_t at;
  int left;  // elements of the entry from here on, at most a chunk's
  float gs, step, rbc2, keep;
  float small_v;  // 8-bit states: blocks with a largest v below take exact roots
};

// A warp's 256 elements lie over its lanes as two groups of 128, four
// neighbours per lane in each, so that a load of fp32 is one run of 512 bytes;
// with 8-bit states, whose codes are a byte each, as eight neighbours per lane.
template <int kBits>
struct Layout {
  static constexpr int kLane = kBits == 8 ? 8 : 4;   // from lane to lane
  static constexpr int kGap = kBits == 8 ? 4 : 128;  // from a lane's first four to its others
};

// With 8-bit states there is enough to compute that a warp's next blocks are
// copied to shared memory ahead (cp.async): each lane copies what it will read
// itself, so nothing waits for another thread and no registers hold what is on
// its way.
template <typename P, typename G>
struct Ahead {
  struct Slot {  // one block of a warp
    P p[32][8];
    G g[32][8];
    uint2 mc[32], rc[32];
  };
  static constexpr int kSlots = sizeof(Slot) <= 2048 ? 3 : 2;  // at most 6 KB per warp
  Slot slot[Step<8>::kWarps][kSlots];
};
template <int kBytes>
__device__ __forceinline__ void copy_ahead(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "n"(kBytes)
               : "memory");
}
template <typename P, typename G>
__device__ __forceinline__ void copy_block(const AdamArgs& a, const Lane<P, G>& e, int tile, typename Ahead<P, G>::Slot& s) {
  const int at = tile * Step<8>::kTile, lane = static_cast<int>(threadIdx.x & 31);
  const int64_t so = e.at + at;
#pragma unroll
  for (int i = 0; i < 8; i += 16 / static_cast<int>(sizeof(G))) copy_ahead<16>(&s.g[lane][i], e.g + at + i);
#pragma unroll
  for (int i = 0; i < 8; i += 16 / static_cast<int>(sizeof(P))) copy_ahead<16>(&s.p[lane][i], e.p + at + i);
  copy_ahead<8>(&s.mc[lane], static_cast<const int8_t*>(a.m) + so);
  copy_ahead<8>(&s.rc[lane], static_cast<const uint8_t*>(a.v) + so);
}

// The warp's 256 elements of a tile. kVec: all there and aligned (with 8-bit
// states, copied ahead, and their scales here). False: a moment has become
// non-finite.
template <typename P, typename G, int kBits, bool kVec>
__device__ __forceinline__ bool step_block(const AdamArgs& a, const Lane<P, G>& e, int tile, const typename Ahead<P, G>::Slot* ahead,
                                           float ms, float rs) {
  constexpr int kGap = Layout<kBits>::kGap;
  const int at = tile * Step<kBits>::kTile, left = e.left - at, lane = static_cast<int>(threadIdx.x & 31);
  const int64_t so = e.at + at;
  float pv[8], gv[8];
  if (kBits == 8 && kVec) {
    near8(ahead->g[lane], gv);
    near8(ahead->p[lane], pv);
  } else {
    load8<kGap, kVec>(e.g + at, left, gv);
    load8<kGap, kVec>(e.p + at, left, pv);
  }
  bool fine;
  if (kBits == 32) {
    float m[8], v[8];
    float *ma = static_cast<float*>(a.m) + so, *va = static_cast<float*>(a.v) + so;
    load8<kGap, true>(ma, 0, m);
    load8<kGap, true>(va, 0, v);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = gv[i] * e.gs;
      m[i] = __fadd_rn(__fmul_rn(m[i], a.b1), __fmul_rn(x, a.one_minus_b1));
      v[i] = __fadd_rn(__fmul_rn(v[i], a.b2), __fmul_rn(__fmul_rn(x, x), a.one_minus_b2));
      const float u = __fdiv_rn(m[i], fmaf(__fsqrt_rn(v[i]), e.rbc2, a.eps));
      pv[i] = fmaf(pv[i], e.keep, -(u * e.step));
      top = max_mag(top, m[i], v[i]);
    }
    fine = top <= FLT_MAX;
    store8<kGap, true>(ma, 0, m);
    store8<kGap, true>(va, 0, v);
  } else {
    uint2* ma = reinterpret_cast<uint2*>(static_cast<int8_t*>(a.m) + so);
    uint2* ra = reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + so);
    if (!kVec) ms = a.m_scale[so / kBlock], rs = a.r_scale[so / kBlock];
    const uint2 mq = kVec ? ahead->mc[lane] : __ldcs(ma), rq = kVec ? ahead->rc[lane] : __ldcs(ra);
    uint32_t mc[2] = {mq.x, mq.y}, rc[2] = {rq.x, rq.y};
    float2 m[4], v[4], r[4];
    float mt = 0.f, vt = 0.f, least = FLT_MAX;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      decode_m4(mc[j], ms, m + 2 * j);
      decode_r4(rc[j], rs, v + 2 * j);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = mul2(make_float2(gv[2 * i], gv[2 * i + 1]), splat(e.gs));
      m[i] = sum2(mul2(m[i], splat(a.b1)), mul2(x, splat(a.one_minus_b1)), a.one);
      v[i] = sum2(mul2(mul2(v[i], v[i]), splat(a.b2)), mul2(mul2(x, x), splat(a.one_minus_b2)), a.one);
      mt = max_mag(mt, m[i].x, m[i].y);
      vt = max_mag(vt, v[i].x, v[i].y);
      least = fminf(least, fminf(v[i].x, v[i].y));
    }
    mt = warp_max_mag(mt), vt = warp_max_mag(vt);
    fine = mt <= FLT_MAX && vt <= FLT_MAX;
    const bool small = vt < e.small_v;
    if (!small) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = make_float2(sqrt_approx(v[i].x), sqrt_approx(v[i].y));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = make_float2(__fsqrt_rn(v[i].x), __fsqrt_rn(v[i].y));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 d = fma2(r[i], splat(e.rbc2), splat(a.eps));
      const float2 u = mul2(mul2(m[i], make_float2(rcp_approx(d.x), rcp_approx(d.y))), splat(-e.step));
      const float2 q = fma2(make_float2(pv[2 * i], pv[2 * i + 1]), splat(e.keep), u);
      pv[2 * i] = q.x, pv[2 * i + 1] = q.y;
    }
    float ms_new = block_scale(mt), rs_new = block_scale(__fsqrt_rn(vt));
    const bool odd_m = !(mt >= kLeastM && mt <= kMostM);
    // zero for blocks held as zero (rcp of their largest would overflow)
    const float mi = ms_new > 0.f ? rcp_approx(mt) * (127.f * 127.f) : 0.f, ri = rs_new > 0.f ? rsqrt_approx(vt) * (255.f * 255.f) : 0.f;
    // a root above zero: a code of at least one
    auto floor_r = [&](float2 k, float2 w) {
      k = make_float2(fmaxf(k.x, 1.f), fmaxf(k.y, 1.f));
      if (least == 0.f) k = make_float2(w.x > 0.f ? k.x : 0.f, w.y > 0.f ? k.y : 0.f);
      return k;
    };
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float2 y[2];
      float worst = 0.f, unused = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 s = mul2(m[2 * j + i], splat(mi));
        y[i] = make_float2(copysignf(sqrt_approx(fabsf(s.x)), s.x), copysignf(sqrt_approx(fabsf(s.y)), s.y));
      }
      mc[j] = pack_codes(y, &worst);
      if (worst > kNearM || odd_m) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 s = m[2 * j + i];
          y[i] = make_float2(copysignf(code_exact(fabsf(s.x), ms_new, 127.f), s.x), copysignf(code_exact(fabsf(s.y), ms_new, 127.f), s.y));
        }
        mc[j] = pack_codes(y, &unused);
      }
      worst = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 s = mul2(r[2 * j + i], splat(ri));
        y[i] = floor_r(make_float2(sqrt_approx(s.x), sqrt_approx(s.y)), v[2 * j + i]);
      }
      rc[j] = pack_codes(y, &worst);
      if (worst > kNearR || small) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 s = v[2 * j + i];
          y[i] = floor_r(make_float2(code_exact(__fsqrt_rn(s.x), rs_new, 255.f), code_exact(__fsqrt_rn(s.y), rs_new, 255.f)), s);
        }
        rc[j] = pack_codes(y, &unused);
      }
    }
    __stcs(ma, make_uint2(mc[0], mc[1]));
    __stcs(ra, make_uint2(rc[0], rc[1]));
    if (!fine) ms_new = rs_new = __int_as_float(0x7fc00000);  // no code says NaN: the block's scale does
    if (lane == 0) a.m_scale[so / kBlock] = ms_new, a.r_scale[so / kBlock] = rs_new;
  }
  store8<kGap, kVec>(e.p + at, left, pv);
  if (e.copy) store8<kGap, kVec>(e.copy + at, left, pv);
  return fine;
}

template <typename P, typename G, int kBits>
__global__ void __launch_bounds__(Step<kBits>::kThreads, Step<kBits>::kPerSm) adamw_kernel(const __grid_constant__ AdamArgs a) {
  pdl_allow_dependents();
  const Chunk c = a.chunks_of[a.chunk0 + blockIdx.x];
  P* p = static_cast<P*>(a.params[c.entry - a.entry0]) + c.first;
  const G* g = static_cast<const G*>(a.grads[c.entry - a.entry0]) + c.first;
  __nv_bfloat16* copy = static_cast<__nv_bfloat16*>(a.copies[c.entry - a.entry0]);
  pdl_wait_predecessor();
  Lane<P, G> e;
  e.gs = 1.f;
  if (a.grad_scale) {
    e.gs = *a.grad_scale;
    if (!(fabsf(e.gs) <= FLT_MAX)) {  // every block sees it: nothing changes, the step does not count
      if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(&a.shared->nonfinite, 0, kSkipped);
      return;
    }
  }
  uint32_t* turn = a.turns + a.chunk0 + blockIdx.x;
  const uint32_t which = *turn;
  const AdamClock* now = a.shared->clock + which;
  e.step = a.lr * now->inv_bc1;
  e.rbc2 = now->inv_sqrt_bc2;
  e.keep = 1.f - a.lr * a.wd * c.decay;
  e.small_v = kLostRoot * e.rbc2 > 0x1p-25f * a.eps ? INFINITY : kSmallV;
  __syncthreads();  // every thread has its turn
  if (threadIdx.x == 0) {
    *turn = which ^ 1u;
    if (a.last && blockIdx.x == 0)
      set_clock(a.shared->clock + (which ^ 1u), now->b1t * a.beta1, now->b2t * a.beta2, now->steps + 1);
  }
  // the lane's first element; the state's arrays are padded to whole blocks
  const int first = static_cast<int>(threadIdx.x >> 5) * kBlock, at = first + Layout<kBits>::kLane * static_cast<int>(threadIdx.x & 31);
  const bool aligned = ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(copy)) & 15u) == 0;
  e.p = p + at, e.g = g + at, e.copy = copy ? copy + c.first + at : nullptr;
  e.at = c.off + at;
  e.left = c.left - at;
  // the warp's tiles that begin in the entry, and those that are whole and aligned
  constexpr int kTile = Step<kBits>::kTile;
  const int left = c.left - first, tiles = left <= 0 ? 0 : (left + kTile - 1) / kTile;
  const int whole = !aligned || tiles == 0 ? 0 : left - (tiles - 1) * kTile >= kBlock ? tiles : tiles - 1;
  bool fine = true;
  if (kBits == 8) {
    using A = Ahead<P, G>;
    __shared__ __align__(16) uint8_t room[kBits == 8 ? sizeof(A) : 16];
    auto& slots = reinterpret_cast<A*>(room)->slot[threadIdx.x >> 5];
    auto ahead = [&](int i, int s) {
      if (i < whole) copy_block(a, e, i, slots[s]);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < A::kSlots - 1; ++s) ahead(s, s);
    int s = 0;
    const float* msp = a.m_scale + e.at / kBlock;
    const float* rsp = a.r_scale + e.at / kBlock;
    float ms = 0.f, rs = 0.f;
    if (whole > 0) ms = *msp, rs = *rsp;
#pragma unroll 1
    for (int i = 0; i < whole; ++i) {
      ahead(i + A::kSlots - 1, s == 0 ? A::kSlots - 1 : s - 1);
      const float ms_now = ms, rs_now = rs;
      if (i + 1 < whole) ms = msp[(i + 1) * (kTile / kBlock)], rs = rsp[(i + 1) * (kTile / kBlock)];
      asm volatile("cp.async.wait_group %0;" ::"n"(A::kSlots - 1) : "memory");
      fine = step_block<P, G, kBits, true>(a, e, i, &slots[s], ms_now, rs_now) && fine;
      if (++s == A::kSlots) s = 0;
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < whole; ++i) fine = step_block<P, G, kBits, true>(a, e, i, nullptr, 0.f, 0.f) && fine;
  }
#pragma unroll 1
  for (int i = whole; i < tiles; ++i) fine = step_block<P, G, kBits, false>(a, e, i, nullptr, 0.f, 0.f) && fine;
  if (!fine) atomicCAS(&a.shared->nonfinite, 0, c.entry + 1);
}

// out[0] = sqrt(sum g^2), out[1] = the coefficient that brings it to at most
// max_norm. Bound by the one read of the gradients, of which a warp takes up to
// 2048 elements at a time. A thread adds the squares
// of its share in fp32 (eight sums side by side), the rest is added as
// WideSum; the blocks' sums lie in `partials` and the last block to finish adds them up,
// in an order that does not depend on which block that is.
template <typename G>
__global__ void __launch_bounds__(kAdamThreads) grad_norm_kernel(const __grid_constant__ NormArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[2][kAdamThreads / 32];
  __shared__ bool final_block;
  constexpr int N = 16 / sizeof(G);  // elements of a 16-byte load
  float2 acc[N / 2] = {};
  const int lane = static_cast<int>(threadIdx.x & 31);
  constexpr int kWarps = kAdamThreads / 32;
  for (int64_t u = blockIdx.x * kWarps + (threadIdx.x >> 5); u < a.chunks << a.shift; u += static_cast<int64_t>(gridDim.x) * kWarps) {
    const Chunk ch = a.chunks_of[a.chunk0 + (u >> a.shift)];
    const int at = static_cast<int>(u - (u >> a.shift << a.shift)) * a.unit, n = min(a.unit, ch.left - at);
    if (n <= 0) continue;
    const G* g = static_cast<const G*>(a.grads[ch.entry - a.entry0]) + ch.first + at;
    // to the next 16-byte boundary one by one, as the rest that fills none at the end
    const int lead = static_cast<int>(((16u - (reinterpret_cast<uintptr_t>(g) & 15u)) & 15u) / sizeof(G));
    const int head = min(lead, n), quads = (n - head) / N;
    if (lane < head) {
      const float x = to_f(g[lane]);
      acc[0].x = fmaf(x, x, acc[0].x);
    }
    const int tail = head + quads * N + lane;
    if (tail < n) {
      const float x = to_f(g[tail]);
      acc[0].y = fmaf(x, x, acc[0].y);
    }
    const uint4* q = reinterpret_cast<const uint4*>(g + head);
#pragma unroll 8
    for (int i = lane; i < quads; i += 32) {
      const uint4 w = __ldcs(q + i);
      G h[N];
      memcpy(h, &w, 16);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const float2 x = make_float2(to_f(h[2 * k]), to_f(h[2 * k + 1]));
        acc[k] = fma2(x, x, acc[k]);
      }
    }
  }
  WideSum t;
#pragma unroll
  for (int k = 0; k < N / 2; ++k) t.add(acc[k].x), t.add(acc[k].y);
  const float s = block_total(t, sh[0]);
  if (threadIdx.x == 0) {
    a.partials[a.part0 + blockIdx.x] = s;
    __threadfence();
    final_block = a.last && atomicInc(&a.shared->norm_ticket, gridDim.x - 1) == gridDim.x - 1;
  }
  __syncthreads();
  if (!final_block) return;
  __threadfence();
  WideSum all;
  for (int i = threadIdx.x; i < a.parts; i += kAdamThreads) all.add(__ldcg(a.partials + i));
  const float total = block_total(all, sh[1]);
  if (threadIdx.x == 0) {
    const float norm = __fsqrt_rn(total);
    a.out[0] = norm;
    a.out[1] = !(norm <= FLT_MAX) ? __int_as_float(0x7fc00000) : norm > a.max_norm ? __fdiv_rn(a.max_norm, norm) : 1.f;
  }
}

// The values that the 8-bit states stand for: two bytes read and eight written
// per element, which bound it. A thread takes four elements.
__global__ void __launch_bounds__(kAdamThreads) adamw_values_kernel(const uint32_t* __restrict__ m_code,
                                                                    const uint32_t* __restrict__ r_code,
                                                                    const float* __restrict__ m_scale,
                                                                    const float* __restrict__ r_scale, int64_t quads,
                                                                    float* __restrict__ m, float* __restrict__ v) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kAdamThreads + threadIdx.x;
  if (i >= quads) return;
  const int64_t b = i / (kBlock / 4);
  float2 x[2];
  if (m) {
    decode_m4(__ldcs(m_code + i), m_scale[b], x);
    __stcs(reinterpret_cast<float4*>(m) + i, make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
  }
  if (v) {
    decode_r4(__ldcs(r_code + i), r_scale[b], x);
    x[0] = mul2(x[0], x[0]), x[1] = mul2(x[1], x[1]);
    __stcs(reinterpret_cast<float4*>(v) + i, make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
  }
}

// One launch's share of the entries.
struct Part {
  int entry0, entries;
  int64_t chunk0, chunks;
  int norm_blocks, part0;
};

size_t dtype_bytes(int t) { return t == MEQ_F32 ? 4 : 2; }

}  // namespace

struct meq_adamw {
  int n = 0;
  std::vector<Part> parts;
  meq_adamw_options opt{};
  int64_t elements = 0;  // of the padded state arrays
  int device = 0, total_parts = 0, norm_shift = 0;
  int64_t chunk = 0;
  char* arena = nullptr;
  void *d_m = nullptr, *d_v = nullptr;
  float *d_ms = nullptr, *d_rs = nullptr;
  Chunk* d_chunks = nullptr;
  uint32_t* d_turns = nullptr;
  AdamShared* d_shared = nullptr;
  float* d_partials = nullptr;
  cudaStream_t last_stream = nullptr;
  bool captured = false;  // a call was captured: replays run on any stream, unseen by the host
  std::string last_error;
};

namespace {

meq_status fail(meq_adamw* st, meq_status s, const std::string& msg) {
  if (st) st->last_error = msg;
  else meq::set_global_error(msg);
  return s;
}
meq_status cuda_fail(meq_adamw* st, cudaError_t e, const char* what) {
  return fail(st, MEQ_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// No C++ exception leaves a C entry.
template <typename F>
meq_status guarded(meq_adamw* st, F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    if (st) st->last_error.clear();
    return MEQ_ERR_OOM;
  } catch (...) {
    return MEQ_ERR_INVALID_ARG;
  }
}

bool valid_adamw_options(const meq_adamw_options& o, std::string* why) {
  auto beta = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!beta(o.beta1) || !beta(o.beta2)) { *why = "beta1 and beta2 must be in [0, 1)"; return false; }
  if (!(static_cast<float>(o.eps) >= FLT_MIN) || !std::isfinite(static_cast<float>(o.eps))) { *why = "eps must be a positive normal number in fp32"; return false; }
  if (o.state_bits != 32 && o.state_bits != 8) { *why = "state_bits must be 32 or 8"; return false; }
  if (o.param_type != MEQ_F32 && o.param_type != MEQ_BF16) { *why = "param_type must be MEQ_F32 or MEQ_BF16"; return false; }
  if (o.grad_type != MEQ_F32 && o.grad_type != MEQ_BF16 && o.grad_type != MEQ_F16) { *why = "grad_type must be a meq_dtype"; return false; }
  return true;
}

int64_t pad_block(int64_t n) { return (n + kBlock - 1) / kBlock * kBlock; }

// Entries, launches and the arena's layout; host only.
struct Plan {
  int64_t elements = 0, chunks = 0, persistent = 0, total = 0;
  int64_t o_m = 0, o_v = 0, o_ms = 0, o_rs = 0, o_chunks = 0, o_turns = 0, o_shared = 0, o_partials = 0;
  int total_parts = 0;
  int64_t chunk = 0;  // elements of one
  int norm_shift = 0;
  std::vector<AdamEntry> entries;
  std::vector<Part> parts;
};
Plan make_plan(const meq_shape* shapes, const float* decay, int n, const meq_adamw_options& o, int sms) {
  Plan P;
  P.entries.resize(n);
  int64_t numel = 0;
  for (int i = 0; i < n; ++i) numel += shapes[i].rows * shapes[i].cols;
  // longer chunks as long as there are some four for every block that the SMs hold
  const bool small = o.state_bits == 8;
  P.chunk = small ? Step<8>::kMinChunk : Step<32>::kMinChunk;
  const int64_t most = small ? Step<8>::kMaxChunk : Step<32>::kMaxChunk;
  const int64_t resident = static_cast<int64_t>(sms) * (small ? Step<8>::kPerSm : Step<32>::kPerSm);
  while (P.chunk < most && numel >= 4 * resident * 2 * P.chunk) P.chunk *= 2;
  while (P.chunk >> P.norm_shift > kNormUnit) ++P.norm_shift;
  for (int i = 0; i < n; ++i) {
    AdamEntry& E = P.entries[i];
    E.numel = shapes[i].rows * shapes[i].cols;
    E.off = P.elements;
    E.chunk0 = P.chunks;
    E.decay = decay ? decay[i] : 1.f;
    P.elements += pad_block(E.numel);
    P.chunks += (E.numel + P.chunk - 1) / P.chunk;
  }
  for (int i = 0; i < n; i += kMaxEntries) {
    Part p{};
    p.entry0 = i;
    p.entries = n - i < kMaxEntries ? n - i : kMaxEntries;
    p.chunk0 = P.entries[i].chunk0;
    p.chunks = (i + p.entries < n ? P.entries[i + p.entries].chunk0 : P.chunks) - p.chunk0;
    const int64_t most = static_cast<int64_t>(sms) * kNormBlocksPerSm;
    const int64_t blocks = ((p.chunks << P.norm_shift) + kAdamThreads / 32 - 1) / (kAdamThreads / 32);
    p.norm_blocks = static_cast<int>(blocks < most ? blocks : most);
    p.part0 = P.total_parts;
    P.total_parts += p.norm_blocks;
    P.parts.push_back(p);
  }
  auto add = [&](int64_t bytes) {
    const int64_t off = P.total;
    P.total += (bytes + 255) / 256 * 256;
    return off;
  };
  const int64_t each = o.state_bits / 8, scales = o.state_bits == 8 ? P.elements / kBlock * 4 : 0;
  P.o_m = add(P.elements * each);
  P.o_v = add(P.elements * each);
  P.o_ms = add(scales);
  P.o_rs = add(scales);
  P.o_chunks = add(P.chunks * static_cast<int64_t>(sizeof(Chunk)));
  P.o_turns = add(P.chunks * 4);
  P.o_shared = add(sizeof(AdamShared));
  P.o_partials = add(static_cast<int64_t>(P.total_parts) * 4);
  P.persistent = 2 * (P.elements * each + scales);
  return P;
}

bool check_plan(const Plan& P, std::string* why) {
  for (const Part& p : P.parts)
    if (p.chunks > 0x7fffffff) { *why = "too many elements in 256 consecutive entries for one launch"; return false; }
  if (P.chunks > 0x7fffffff) { *why = "more than 2^42 elements in one state"; return false; }
  return true;
}

meq_status check_call(meq_adamw* st, const void* const* ptrs, size_t align, const char* what) {
  if (!ptrs) return fail(st, MEQ_ERR_INVALID_ARG, std::string(what) + " must be non-NULL");
  for (int i = 0; i < st->n; ++i) {
    if (!ptrs[i]) return fail(st, MEQ_ERR_INVALID_ARG, std::string("NULL ") + what + " pointer at " + std::to_string(i));
    if (reinterpret_cast<uintptr_t>(ptrs[i]) % align)
      return fail(st, MEQ_ERR_INVALID_ARG, std::string(what) + " pointer " + std::to_string(i) + " is not aligned to its type");
  }
  return MEQ_OK;
}

meq_status check_device(meq_adamw* st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(st, e, "cudaGetDevice");
  if (dev != st->device)
    return fail(st, MEQ_ERR_INVALID_ARG, "the state is on device " + std::to_string(st->device) + ", the current device is " + std::to_string(dev));
  return MEQ_OK;
}

// What the state's calls wait for: the stream of the last one, and of a state
// whose calls were captured, whose replays do not pass here, the whole device.
void enqueued(meq_adamw* st, cudaStream_t s) {
  st->last_stream = s;
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &status) != cudaSuccess) cudaGetLastError();
  if (status != cudaStreamCaptureStatusNone) st->captured = true;
}
cudaError_t wait_for_all(meq_adamw* st) {
  if (!st->captured) return cudaStreamSynchronize(st->last_stream);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev != st->device) e = cudaSetDevice(st->device);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (dev != st->device) cudaSetDevice(dev);
  return e;
}

template <typename P, typename G>
cudaError_t launch_adamw(int bits, const AdamArgs& a, unsigned grid, cudaStream_t s) {
  if (bits == 32) return launch_pdl(adamw_kernel<P, G, 32>, dim3(grid), dim3(Step<32>::kThreads), 0, s, 1, a);
  return launch_pdl(adamw_kernel<P, G, 8>, dim3(grid), dim3(Step<8>::kThreads), 0, s, 1, a);
}
template <typename P>
cudaError_t launch_adamw(const meq_adamw_options& o, const AdamArgs& a, unsigned grid, cudaStream_t s) {
  if (o.grad_type == MEQ_F32) return launch_adamw<P, float>(o.state_bits, a, grid, s);
  if (o.grad_type == MEQ_BF16) return launch_adamw<P, __nv_bfloat16>(o.state_bits, a, grid, s);
  return launch_adamw<P, __half>(o.state_bits, a, grid, s);
}

}  // namespace

extern "C" {

void meq_adamw_default_options(meq_adamw_options* opt) {
  if (!opt) return;
  std::memset(opt, 0, sizeof(*opt));
  opt->beta1 = 0.9, opt->beta2 = 0.999, opt->eps = 1e-8;
  opt->state_bits = 32;
  opt->param_type = MEQ_F32, opt->grad_type = MEQ_F32;
}

meq_status meq_adamw_state_bytes(const meq_shape* shapes, int n, const meq_adamw_options* opt, size_t* persistent_bytes,
                                 size_t* workspace_bytes) {
  return guarded(nullptr, [&]() -> meq_status {
    meq_adamw_options o;
    if (opt) o = *opt; else meq_adamw_default_options(&o);
    std::string why;
    if (!meq::valid_shapes(shapes, n, &why) || !valid_adamw_options(o, &why)) return fail(nullptr, MEQ_ERR_INVALID_ARG, why);
    const Plan P = make_plan(shapes, nullptr, n, o, 152);
    if (!check_plan(P, &why)) return fail(nullptr, MEQ_ERR_INVALID_ARG, why);
    if (persistent_bytes) *persistent_bytes = static_cast<size_t>(P.persistent);
    if (workspace_bytes) *workspace_bytes = static_cast<size_t>(P.total - P.persistent);
    return MEQ_OK;
  });
}

meq_status meq_adamw_init(const meq_shape* shapes, const float* decay, int n, const meq_adamw_options* opt,
                          void* cuda_stream, meq_adamw** out) {
  if (!out) return fail(nullptr, MEQ_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  return guarded(nullptr, [&]() -> meq_status {
    meq_adamw_options o;
    if (opt) o = *opt; else meq_adamw_default_options(&o);
    std::string why;
    if (!meq::valid_shapes(shapes, n, &why) || !valid_adamw_options(o, &why)) return fail(nullptr, MEQ_ERR_INVALID_ARG, why);
    for (int i = 0; decay && i < n; ++i)
      if (!(decay[i] >= 0.f) || !std::isfinite(decay[i]))
        return fail(nullptr, MEQ_ERR_INVALID_ARG, "decay of entry " + std::to_string(i) + " must be finite and >= 0");
    int dev = 0, sms = 0;
    meq_status ms = meq::check_sm103(&dev, &sms);
    if (ms != MEQ_OK) return ms;
    Plan P = make_plan(shapes, decay, n, o, sms);
    if (!check_plan(P, &why)) return fail(nullptr, MEQ_ERR_INVALID_ARG, why);
    const int64_t size = P.chunk;
    std::vector<Chunk> chunks;
    chunks.reserve(static_cast<size_t>(P.chunks));
    for (int i = 0; i < n; ++i) {
      const AdamEntry& E = P.entries[i];
      for (int64_t at = 0; at < E.numel; at += size)
        chunks.push_back(Chunk{at, E.off + at, static_cast<int32_t>(E.numel - at < size ? E.numel - at : size), i, E.decay, 0});
    }
    AdamClock clock[2];
    set_clock(clock, o.beta1, o.beta2, 0);
    clock[1] = clock[0];

    struct Owner {  // of the state until it is handed out
      meq_adamw* st;
      ~Owner() {
        if (!st) return;
        if (st->arena) cudaFree(st->arena);
        delete st;
      }
    } own{new meq_adamw()};
    meq_adamw* st = own.st;
    st->n = n, st->opt = o, st->device = dev;
    st->elements = P.elements, st->total_parts = P.total_parts, st->norm_shift = P.norm_shift, st->chunk = P.chunk;
    cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&st->arena), static_cast<size_t>(P.total));
    if (e != cudaSuccess) {
      cudaGetLastError();
      st->arena = nullptr;
      return fail(nullptr, MEQ_ERR_OOM, "cudaMalloc of " + std::to_string(P.total) + " bytes failed");
    }
    char* A = st->arena;
    st->d_m = A + P.o_m, st->d_v = A + P.o_v;
    st->d_ms = reinterpret_cast<float*>(A + P.o_ms), st->d_rs = reinterpret_cast<float*>(A + P.o_rs);
    st->d_chunks = reinterpret_cast<Chunk*>(A + P.o_chunks);
    st->d_turns = reinterpret_cast<uint32_t*>(A + P.o_turns);
    st->d_shared = reinterpret_cast<AdamShared*>(A + P.o_shared);
    st->d_partials = reinterpret_cast<float*>(A + P.o_partials);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    e = cudaMemsetAsync(A, 0, static_cast<size_t>(P.total), s);
    if (e == cudaSuccess) e = cudaMemcpyAsync(st->d_chunks, chunks.data(), sizeof(Chunk) * chunks.size(), cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaMemcpyAsync(st->d_shared->clock, clock, sizeof(clock), cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return fail(nullptr, MEQ_ERR_CUDA, std::string("initialising the AdamW state failed: ") + cudaGetErrorString(e));
    st->parts = std::move(P.parts);
    st->last_stream = s;
    own.st = nullptr;
    *out = st;
    return MEQ_OK;
  });
}

meq_status meq_adamw_grad_norm(const void* const* grads, meq_adamw* st, float max_norm, float* out, void* cuda_stream) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    meq_status ms = check_call(st, grads, dtype_bytes(st->opt.grad_type), "grads");
    if (ms != MEQ_OK) return ms;
    if (!out || reinterpret_cast<uintptr_t>(out) % 4) return fail(st, MEQ_ERR_INVALID_ARG, "out must be a device pointer to two floats");
    if (!(max_norm > 0.f)) return fail(st, MEQ_ERR_INVALID_ARG, "max_norm must be > 0");
    ms = check_device(st);
    if (ms != MEQ_OK) return ms;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    NormArgs a;
    a.chunks_of = st->d_chunks, a.shared = st->d_shared, a.partials = st->d_partials;
    a.out = out, a.max_norm = max_norm, a.parts = st->total_parts;
    a.shift = st->norm_shift, a.unit = static_cast<int32_t>(st->chunk >> st->norm_shift);
    for (size_t k = 0; k < st->parts.size(); ++k) {
      const Part& p = st->parts[k];
      a.entry0 = p.entry0, a.chunk0 = p.chunk0, a.chunks = p.chunks, a.part0 = p.part0;
      a.last = k + 1 == st->parts.size() ? 1 : 0;
      for (int i = 0; i < p.entries; ++i) a.grads[i] = grads[p.entry0 + i];
      const dim3 grid(static_cast<unsigned>(p.norm_blocks)), block(kAdamThreads);
      cudaError_t e = st->opt.grad_type == MEQ_F32    ? launch_pdl(grad_norm_kernel<float>, grid, block, 0, s, 1, a)
                      : st->opt.grad_type == MEQ_BF16 ? launch_pdl(grad_norm_kernel<__nv_bfloat16>, grid, block, 0, s, 1, a)
                                                      : launch_pdl(grad_norm_kernel<__half>, grid, block, 0, s, 1, a);
      if (e != cudaSuccess) return cuda_fail(st, e, "gradient norm launch");
    }
    enqueued(st, s);
    return MEQ_OK;
  });
}

meq_status meq_adamw_step(void* const* params, const void* const* grads, void* const* copies, meq_adamw* st, float lr,
                          float weight_decay, const float* grad_scale, void* cuda_stream) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    meq_status ms = check_call(st, const_cast<const void* const*>(params), dtype_bytes(st->opt.param_type), "params");
    if (ms == MEQ_OK) ms = check_call(st, grads, dtype_bytes(st->opt.grad_type), "grads");
    if (ms == MEQ_OK && copies) ms = check_call(st, const_cast<const void* const*>(copies), 2, "copies");
    if (ms != MEQ_OK) return ms;
    if (!std::isfinite(lr) || !std::isfinite(weight_decay)) return fail(st, MEQ_ERR_INVALID_ARG, "lr and weight_decay must be finite");
    if (reinterpret_cast<uintptr_t>(grad_scale) % 4) return fail(st, MEQ_ERR_INVALID_ARG, "grad_scale is not aligned to its type");
    ms = check_device(st);
    if (ms != MEQ_OK) return ms;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    AdamArgs a;
    a.chunks_of = st->d_chunks, a.turns = st->d_turns, a.shared = st->d_shared;
    a.m = st->d_m, a.v = st->d_v, a.m_scale = st->d_ms, a.r_scale = st->d_rs, a.grad_scale = grad_scale;
    a.beta1 = st->opt.beta1, a.beta2 = st->opt.beta2;
    a.b1 = static_cast<float>(a.beta1), a.one_minus_b1 = static_cast<float>(1.0 - a.beta1);
    a.b2 = static_cast<float>(a.beta2), a.one_minus_b2 = static_cast<float>(1.0 - a.beta2);
    a.eps = static_cast<float>(st->opt.eps), a.lr = lr, a.wd = weight_decay, a.one = 1.f;
    for (size_t k = 0; k < st->parts.size(); ++k) {
      const Part& p = st->parts[k];
      a.entry0 = p.entry0, a.chunk0 = p.chunk0;
      a.last = k + 1 == st->parts.size() ? 1 : 0;
      for (int i = 0; i < p.entries; ++i) {
        a.params[i] = params[p.entry0 + i];
        a.grads[i] = grads[p.entry0 + i];
        a.copies[i] = copies ? copies[p.entry0 + i] : nullptr;
      }
      const unsigned grid = static_cast<unsigned>(p.chunks);
      cudaError_t e = st->opt.param_type == MEQ_F32 ? launch_adamw<float>(st->opt, a, grid, s)
                                                    : launch_adamw<__nv_bfloat16>(st->opt, a, grid, s);
      if (e != cudaSuccess) return cuda_fail(st, e, "AdamW launch");
    }
    enqueued(st, s);
    return MEQ_OK;
  });
}

meq_status meq_adamw_state_ptrs(meq_adamw* st, void** m, void** v, float** m_scale, float** v_scale, int64_t* elements) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  const bool scales = st->opt.state_bits == 8;
  if (m) *m = st->d_m;
  if (v) *v = st->d_v;
  if (m_scale) *m_scale = scales ? st->d_ms : nullptr;
  if (v_scale) *v_scale = scales ? st->d_rs : nullptr;
  if (elements) *elements = st->elements;
  return MEQ_OK;
}

meq_status meq_adamw_read_values(meq_adamw* st, float* m, float* v, void* cuda_stream) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    if ((reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(v)) % 16)
      return fail(st, MEQ_ERR_INVALID_ARG, "m and v must be 16-byte aligned");
    meq_status ms = check_device(st);
    if (ms != MEQ_OK) return ms;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = cudaSuccess;
    if (st->opt.state_bits == 32) {
      const size_t bytes = static_cast<size_t>(st->elements) * 4;
      if (m) e = cudaMemcpyAsync(m, st->d_m, bytes, cudaMemcpyDeviceToDevice, s);
      if (e == cudaSuccess && v) e = cudaMemcpyAsync(v, st->d_v, bytes, cudaMemcpyDeviceToDevice, s);
    } else if (m || v) {
      const int64_t quads = st->elements / 4, blocks = (quads + kAdamThreads - 1) / kAdamThreads;
      e = launch_pdl(adamw_values_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kAdamThreads), 0, s, 1,
                     static_cast<const uint32_t*>(st->d_m), static_cast<const uint32_t*>(st->d_v),
                     static_cast<const float*>(st->d_ms), static_cast<const float*>(st->d_rs), quads, m, v);
    }
    if (e != cudaSuccess) return cuda_fail(st, e, "reading the AdamW state");
    enqueued(st, s);
    return MEQ_OK;
  });
}

meq_status meq_adamw_steps(meq_adamw* st, int64_t* steps) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    if (!steps) return fail(st, MEQ_ERR_INVALID_ARG, "steps is NULL");
    AdamClock c[2];
    cudaError_t e = wait_for_all(st);
    if (e == cudaSuccess) e = cudaMemcpy(c, st->d_shared->clock, sizeof(c), cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return cuda_fail(st, e, "reading the step count");
    *steps = c[0].steps > c[1].steps ? c[0].steps : c[1].steps;  // the next step's is the later one
    return MEQ_OK;
  });
}

meq_status meq_adamw_set_steps(meq_adamw* st, int64_t steps) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    if (steps < 0) return fail(st, MEQ_ERR_INVALID_ARG, "steps must be >= 0");
    AdamClock c[2];  // alike, whichever the next step reads
    set_clock(c, std::pow(st->opt.beta1, static_cast<double>(steps) + 1.0),
              std::pow(st->opt.beta2, static_cast<double>(steps) + 1.0), steps);
    c[1] = c[0];
    cudaError_t e = wait_for_all(st);
    if (e == cudaSuccess) e = cudaMemcpy(st->d_shared->clock, c, sizeof(c), cudaMemcpyHostToDevice);
    if (e != cudaSuccess) return cuda_fail(st, e, "writing the step count");
    return MEQ_OK;
  });
}

meq_status meq_adamw_sync(meq_adamw* st) {
  if (!st) return fail(nullptr, MEQ_ERR_INVALID_ARG, "state is NULL");
  return guarded(st, [&]() -> meq_status {
    cudaError_t e = wait_for_all(st);
    if (e != cudaSuccess) return cuda_fail(st, e, "waiting for the state's work");
    int bad = 0;
    e = cudaMemcpy(&bad, &st->d_shared->nonfinite, sizeof(int), cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return cuda_fail(st, e, "reading the non-finite flag");
    if (bad == 0) return MEQ_OK;
    const int zero = 0;
    e = cudaMemcpy(&st->d_shared->nonfinite, &zero, sizeof(int), cudaMemcpyHostToDevice);
    if (e != cudaSuccess) return cuda_fail(st, e, "clearing the non-finite flag");
    if (bad == kSkipped) return fail(st, MEQ_ERR_NONFINITE, "a step was skipped: its gradient coefficient was not finite");
    return fail(st, MEQ_ERR_NONFINITE, "non-finite moment (gradient, or a previous non-finite step) in entry " + std::to_string(bad - 1));
  });
}

meq_status meq_adamw_free(meq_adamw* st) {
  if (!st) return MEQ_OK;
  wait_for_all(st);
  if (st->arena) cudaFree(st->arena);
  delete st;
  return MEQ_OK;
}

const char* meq_adamw_last_error(const meq_adamw* st) { return st ? st->last_error.c_str() : meq_last_error(nullptr); }

}  // extern "C"

// Rows of activations on their way through the norms' persistent kernels: how a
// row is shared out to threads, copied ahead into shared memory, and reduced.
//
// A group of `warps` warps takes a row at a time, each warp consecutive columns
// of it; of short rows a warp takes several at once, `lanes` lanes each. Piece k
// of a lane is 16 bytes' worth of columns, the same ones in every row, so weights
// stay in registers, and so do the sums over rows of the weight's gradient.
//
// Rows are copied into a ring of slots (cp.async) `depth` - 1 rows ahead, which
// keeps enough bytes on their way whatever the registers leave of the
// occupancy; a thread copies the pieces that it reads itself, and no thread waits
// for another.
//
// Rows that start elsewhere in their 16 bytes (kOffset): the grid is a multiple of
// 8 blocks, so the rows of one thread all start at the same place in them, and its
// pieces are cut at 16-byte boundaries once for all rows. Only a row's first and
// last piece may be a part, which is stored element by element. (Pieces cut from
// the row's start, shifted into place on the way in and out, took 2 to 3 times the
// time: 16384 x 2047 bf16 forward 52 us, 40 so; backward 151 and 67.)
#pragma once

#include "meq_call.cuh"
#include "meq_mbar.cuh"
#include "norms.cuh"

namespace meq {
namespace norm {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMostDepth = 4;
constexpr int kRingBudget = 220 * 1024;

struct RowShape {
  int lanes;       // of a warp, for a row: a power of two; 32 when a row takes whole warps
  int warps;       // of a row's group (1 when lanes < 32)
  int groups;      // of a block
  int depth;       // slots of a row's ring
  int slot_bytes;  // of one matrix's row, or a warp's part of it
};

// The partial sums of a block's warps, those of a group in 16-byte words (zeros where it has fewer).
constexpr int kMostSums = 64;
struct Exchange {
  float4 sum[2][2][kMostSums / 4];  // two in turn, of two values
};

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// The oldest of depth - 1 rows under way has arrived (this thread's part of it).
__device__ __forceinline__ void copies_wait(int depth) {
  if (depth == 4) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (depth == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A thread's place in its rows.
template <typename T, int kPieces, bool kOffset>
struct Place {
  static constexpr int N = Elem<T>::N, H = kPieces * N / 2, W = N / 2;  // pairs of elements: of a thread, of a piece
  int lanes, lane, group, sub, warp_in;
  int lead;   // elements of the rows' first 16 bytes that precede them
  int begin;  // column of the thread's first element (-lead for the first thread's)
  int left;   // columns from there to the row's end (negative: it has none)
  __device__ __forceinline__ explicit Place(const RowShape& s) {
    const int warp = static_cast<int>(threadIdx.x >> 5);
    lanes = kPieces > 1 ? 32 : s.lanes;
    lane = static_cast<int>(threadIdx.x & 31) & (lanes - 1);
    sub = static_cast<int>(threadIdx.x & 31) / lanes;
    group = warp / s.warps;
    warp_in = warp - group * s.warps;
  }
  // `row`: any of the thread's rows.
  __device__ __forceinline__ void set(const void* base, uint32_t row, int64_t ld, int64_t cols) {
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) + row * static_cast<uint32_t>(ld) * static_cast<uint32_t>(sizeof(T));
    lead = kOffset ? static_cast<int>((at & 15) / sizeof(T)) : 0;
    begin = (warp_in * 32 * kPieces + lane) * N - lead;
    left = static_cast<int>(cols) - begin;
  }
  // Column of piece k's first element, from `begin`.
  __device__ __forceinline__ int col(int k) const { return k * lanes * N; }
  __device__ __forceinline__ bool has(int k) const { return col(k) < left; }
  // Whether the row starts or ends inside piece k.
  __device__ __forceinline__ bool part(int k) const {
    return kOffset && ((k == 0 && begin < 0) || static_cast<unsigned>(left - col(k) - 1) < static_cast<unsigned>(N - 1));
  }
  __device__ __forceinline__ bool exists(int k, int e) const { return (!kOffset || k > 0 || begin + e >= 0) && col(k) + e < left; }
  // The thread's first element of a row.
  __device__ __forceinline__ T* at(const void* base, uint32_t row, int64_t ld) const {
    return const_cast<T*>(static_cast<const T*>(base)) + (static_cast<int64_t>(static_cast<uint64_t>(row) * static_cast<uint64_t>(ld)) + begin);
  }

  // Starts the copies of the thread's pieces of a matrix's row into a slot.
  __device__ __forceinline__ void copy(uint32_t slot, const void* base, uint32_t row, int64_t ld, int64_t rows, int64_t cols) const {
    const T* p = at(base, row, ld);
    slot += static_cast<uint32_t>(lane) * 16u;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if (!has(k)) continue;
      if (part(k)) copy_part(slot + static_cast<uint32_t>(k * lanes) * 16u, p + col(k), base, ld, rows, cols);
      else copy_async16(slot + static_cast<uint32_t>(k * lanes) * 16u, p + col(k));
    }
  }
  // 16 bytes that belong to the row in part: element by element where they reach beyond the matrix.
  static __device__ __noinline__ void copy_part(uint32_t slot, const T* p, const void* base, int64_t ld, int64_t rows, int64_t cols) {
    const T *lo = static_cast<const T*>(base), *hi = lo + ((rows - 1) * ld + cols);
    if (p >= lo && p + N <= hi) {
      copy_async16(slot, p);
      return;
    }
#pragma unroll 1
    for (int e = 0; e < N; ++e) {
      if (p + e < lo || p + e >= hi) continue;
      const uint32_t bits = *reinterpret_cast<const typename Elem<T>::Bits*>(p + e);
      if (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(slot + 4 * e), "r"(bits) : "memory");
      else asm volatile("st.shared.u16 [%0], %1;" ::"r"(slot + 2 * e), "h"(static_cast<uint16_t>(bits)) : "memory");
    }
  }
  // Zeroes a slot's pieces that no copy ever fills.
  __device__ __forceinline__ void clear_slot(uint8_t* slot) const {
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      if (!has(k)) reinterpret_cast<uint4*>(slot)[lane + k * lanes] = make_uint4(0, 0, 0, 0);
  }
  // Piece k of a row in a slot; 0 beyond the row. Rows that a warp takes alone all exist (`in`).
  __device__ __forceinline__ void read(const uint8_t* slot, int k, bool in, float2 (&x)[W]) const {
    uint4 q = reinterpret_cast<const uint4*>(slot)[lane + k * lanes];
    if (kPieces == 1 && !in) q = make_uint4(0, 0, 0, 0);
    Elem<T>::unpack(q, x);
    if (part(k)) clip(k, x);
  }
  // Sets the elements beyond the row to zero.
  __device__ __forceinline__ void clip(int k, float2* x) const {
#pragma unroll
    for (int e = 0; e < W; ++e) {
      if (!exists(k, 2 * e)) x[e].x = 0.f;
      if (!exists(k, 2 * e + 1)) x[e].y = 0.f;
    }
  }
  // Writes piece k; row: the thread's first element.
  __device__ __forceinline__ void write(T* row, int k, const float2* x) const {
    if (!has(k)) return;
    const uint4 q = Elem<T>::pack(x);
    if (!part(k)) {
      *reinterpret_cast<uint4*>(row + col(k)) = q;
      return;
    }
    // Part of 16 bytes: two, four and eight of them at a time, each at its own alignment.
    uint8_t* p = reinterpret_cast<uint8_t*>(row + col(k));
    const int from = k == 0 && begin < 0 ? -begin * static_cast<int>(sizeof(T)) : 0;
    const int to = min((left - col(k)) * static_cast<int>(sizeof(T)), 16);
    if (from > 0 && to < 16) {  // a row within 16 bytes
      using Bits = typename Elem<T>::Bits;
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (exists(k, e)) reinterpret_cast<Bits*>(p)[e] = static_cast<Bits>(sizeof(T) == 4 ? w[e % 4] : w[e / 2] >> (e % 2 * 16));
    } else if (from > 0) {
      int at = from;
      if (sizeof(T) == 2 && (at & 2)) {
        *reinterpret_cast<uint16_t*>(p + at) = static_cast<uint16_t>((at & 8 ? (at & 4 ? q.w : q.z) : at & 4 ? q.y : q.x) >> 16);
        at += 2;
      }
      if (at & 4) {
        *reinterpret_cast<uint32_t*>(p + at) = at & 8 ? q.w : q.y;
        at += 4;
      }
      if (at & 8) *reinterpret_cast<uint2*>(p + 8) = make_uint2(q.z, q.w);
    } else {
      if (to & 8) *reinterpret_cast<uint2*>(p) = make_uint2(q.x, q.y);
      if (to & 4) *reinterpret_cast<uint32_t*>(p + (to & 8)) = to & 8 ? q.z : q.x;
      if (sizeof(T) == 2 && (to & 2))
        *reinterpret_cast<uint16_t*>(p + (to & 12)) = static_cast<uint16_t>(to & 8 ? (to & 4 ? q.w : q.z) : to & 4 ? q.y : q.x);
    }
  }
  // A vector's elements at the thread's columns (0 beyond the row, `none` without a vector).
  __device__ __forceinline__ void vector(const void* v, int type, float none, float2 (&x)[H]) const {
    if (!v) {
#pragma unroll
      for (int i = 0; i < H; ++i) x[i] = make_float2(none, none);
    } else if (type == MEQ_F32) {  // outside the loops: the loads of all elements are on their way together
      vector_of(static_cast<const float*>(v), x);
    } else if (type == MEQ_BF16) {
      vector_of(static_cast<const __nv_bfloat16*>(v), x);
    } else {
      vector_of(static_cast<const __half*>(v), x);
    }
  }
  template <typename V>
  __device__ __forceinline__ void vector_of(const V* v, float2 (&x)[H]) const {
    constexpr int kLoads = N / Elem<V>::N > 0 ? N / Elem<V>::N : 1;  // 16-byte loads per piece
    if (!kOffset && N >= Elem<V>::N && (reinterpret_cast<uintptr_t>(v) & 15) == 0) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
          uint4 q = make_uint4(0, 0, 0, 0);
          if (has(k)) q = *reinterpret_cast<const uint4*>(v + begin + col(k) + l * Elem<V>::N);
          Elem<V>::unpack(q, x + k * W + l * Elem<V>::N / 2);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = i / W, e = 2 * (i % W);
      x[i].x = exists(k, e) ? Elem<V>::get(v + begin + col(k) + e) : 0.f;
      x[i].y = exists(k, e + 1) ? Elem<V>::get(v + begin + col(k) + e + 1) : 0.f;
    }
  }
};

__device__ __forceinline__ void group_barrier(const RowShape& s, int group) {
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * s.warps) : "memory");
}

__device__ __forceinline__ void clear(Exchange& ex) {
  float* p = reinterpret_cast<float*>(&ex);
  for (int i = static_cast<int>(threadIdx.x); i < 4 * kMostSums; i += static_cast<int>(blockDim.x)) p[i] = 0.f;
  __syncthreads();
}
// kValues sums over a row's threads, for each of them, in a fixed order. `turn`
// alternates between calls: a warp may be one call ahead of its group.
template <int kValues, bool kWarp, typename P>
__device__ __forceinline__ void row_sum(float (&v)[kValues], const RowShape& s, const P& p, Exchange& ex, int& turn) {
  if (kWarp) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < kValues; ++i) v[i] += __shfl_xor_sync(kFull, v[i], o);
    }
  } else {
    for (int o = s.lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < kValues; ++i) v[i] += __shfl_xor_sync(kFull, v[i], o);
    }
  }
  if (s.warps == 1) return;
  const int words = (s.warps + 3) / 4;
#pragma unroll
  for (int i = 0; i < kValues; ++i)
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float*>(ex.sum[turn][i] + p.group * words)[p.warp_in] = v[i];
  group_barrier(s, p.group);
#pragma unroll
  for (int i = 0; i < kValues; ++i) {
    const float4* q = ex.sum[turn][i] + p.group * words;
    float4 t = q[0];
    for (int w = 1; w < words; ++w) {
      const float4 u = q[w];
      t.x += u.x, t.y += u.y, t.z += u.z, t.w += u.w;
    }
    v[i] = (t.x + t.y) + (t.z + t.w);
  }
  turn ^= 1;
}

// Both rounded to T and widened again.
template <typename T>
__device__ __forceinline__ float2 round_pair(float2 x) {
  const T a = Elem<T>::make(x.x), b = Elem<T>::make(x.y);
  return make_float2(Elem<T>::get(&a), Elem<T>::get(&b));
}

// ------------------------------------------------------------------- host
constexpr int kMostPieces = 4;  // per thread
constexpr int kMostCluster = 8; // blocks that add up the sums over few rows among themselves
constexpr int kMostHeld = 16;   // elements of a thread that keeps two sums of each and the weights in registers

// Whether the rows of the matrices (NULL: none) lie in their 16 bytes alike; offset: they do not all start there.
template <typename T>
struct Starts {
  bool alike = true, offset = false;
  uintptr_t base = 0, step = 0;
  bool any = false;
  void add(const void* p, int64_t ld, int64_t rows) {
    if (!p) return;
    const uintptr_t b = reinterpret_cast<uintptr_t>(p) % 16, s = rows > 1 ? static_cast<uintptr_t>(ld) * sizeof(T) % 16 : 0;
    alike = alike && (!any || (b == base && s == step));
    base = b, step = s, any = true;
    offset = offset || b != 0 || s != 0;
  }
};

// Warps of a block, by the registers that a thread's elements leave.
inline int most_warps(int elements) { return elements > 16 ? 16 : elements > 8 ? 20 : 32; }

// How rows of `cols` elements, n of them to a piece, are shared out, with `matrices` copied per row. False: they
// are too long. two_sums: a thread keeps two sums per element.
inline bool row_shape(int64_t cols, int n, bool offset, int matrices, bool two_sums, RowShape* s, int* pieces) {
  const int64_t units = (cols + (offset ? n - 1 : 0) + n - 1) / n;  // at most, wherever a row starts
  s->lanes = 32, s->warps = 1, *pieces = 1;
  if (units <= 16) {
    s->lanes = 1;
    while (s->lanes < units) s->lanes *= 2;
  } else {
    // Instructions per row: a warp's pieces, whether they exist or not, and about as many as one piece takes beside them.
    int64_t least = INT64_MAX;
    for (int k = kMostPieces; k >= 1; --k) {
      const int64_t warps = (units + 32 * k - 1) / (32 * k);
      // 32 elements with their weights and two sums spill (8192 x 5461 bf16, backward: 143 us; 24 of them: 87)
      if (offset && two_sums && n * k > 24 && units <= 32 * 3 * most_warps(n * 3)) continue;
      if (warps > most_warps(n * k) || warps * (k + 1) >= least) continue;
      least = warps * (k + 1);
      s->warps = static_cast<int>(warps), *pieces = k;
    }
    if (least == INT64_MAX) return false;
  }
  s->groups = most_warps(n * *pieces) / s->warps;
  if (s->warps > 1 && s->groups > 15) s->groups = 15;  // named barriers
  s->slot_bytes = s->lanes * *pieces * 16;
  // the weights, where they lie beside the ring
  const int weight_bytes = two_sums && !offset && n * *pieces > kMostHeld ? s->warps * s->lanes * *pieces * n * 4 : 0;
  auto fits = [&](int depth) {
    return static_cast<int64_t>(s->groups) * s->warps * (32 / s->lanes) * depth * matrices * s->slot_bytes + weight_bytes <= kRingBudget;
  };
  while (s->groups > 1 && !fits(2)) --s->groups;
  if (!fits(2)) return false;
  s->depth = kMostDepth;
  while (!fits(s->depth)) --s->depth;
  return true;
}
// Blocks for `sets` of rows: with an offset a multiple of 8, so that a thread's rows lie in their 16 bytes alike.
inline unsigned blocks_for(int64_t sets, int sms, bool offset) {
  const int64_t n = sets < sms ? sets : sms;
  return static_cast<unsigned>(!offset ? n : n < sms || sms < 8 ? (n + 7) / 8 * 8 : n / 8 * 8);
}
__host__ __device__ inline int ring_bytes(const RowShape& s, int matrices) {
  return s.groups * s.warps * (32 / s.lanes) * s.depth * matrices * s.slot_bytes;
}

// Shapes and launches, in files of their own. False: the rows are too long, nothing was launched.
bool launch_row_forward(const ForwardArgs& a, int type, int sms, cudaStream_t st, cudaError_t* e);
bool launch_row_backward(const BackwardArgs& a, int type, bool layer, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e);
// The same on few rows by one cluster, which writes dweight and dbias.
bool launch_few_backward(const BackwardArgs& a, int type, bool layer, cudaStream_t st, cudaError_t* e);

}  // namespace norm
}  // namespace meq

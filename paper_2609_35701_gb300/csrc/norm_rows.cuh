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
// occupancy. Where every row starts at 16 bytes a thread copies the pieces that
// it reads itself, and no thread waits for another. Else (kShifted) a warp copies
// the 16-byte words that hold its columns, a lane's piece is shifted out of two
// of them, and pieces are shifted back into words, with the neighbour lane's, to
// be stored: nothing but the ends of a warp's columns goes element by element.
#pragma once

#include <map>
#include <mutex>

#include "meq_mbar.cuh"
#include "norms.cuh"

namespace meq {
namespace norm {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMostDepth = 4;
constexpr int kMostWarps = 32;
constexpr int kRingBudget = 220 * 1024;

struct RowShape {
  int lanes;       // of a warp, for a row: a power of two; 32 when a row takes whole warps
  int warps;       // of a row's group (1 when lanes < 32)
  int groups;      // of a block
  int depth;       // slots of a row's ring
  int slot_bytes;  // of one matrix's row, or a warp's part of it
};

// The partial sums of a block's warps.
struct Exchange {
  float2 sum[2][kMostWarps];
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

// Bytes `from` .. `from` + 15 of the 32 bytes of a and b (from: a multiple of the element's size, at most 16).
template <typename T>
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int from) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (from & 16) {
    return b;
  }
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = from & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = from & 4 ? w[i + 1] : w[i];
  if (sizeof(T) == 2) {
    const int bits = (from & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A thread's place in its row.
template <typename T, int kPieces, bool kShifted>
struct Place {
  static constexpr int N = Elem<T>::N, H = kPieces * N / 2, W = N / 2;  // pairs of elements: of a thread, of a piece
  int lanes, lane, group, sub, warp_in;
  int left;  // columns from the thread's first one to the row's end (negative: it has none)
  int segment, segment_bytes;  // the warp's first column, and the bytes of its columns
  __device__ __forceinline__ Place(const RowShape& s, int64_t cols) {
    const int warp = static_cast<int>(threadIdx.x >> 5);
    lanes = kPieces > 1 ? 32 : s.lanes;
    lane = static_cast<int>(threadIdx.x & 31) & (lanes - 1);
    sub = static_cast<int>(threadIdx.x & 31) / lanes;
    group = warp / s.warps;
    warp_in = warp - group * s.warps;
    segment = warp_in * 32 * kPieces * N;
    const int rest = static_cast<int>(cols) - segment;
    left = rest - lane * N;
    segment_bytes = max(0, min(rest, lanes * kPieces * N)) * static_cast<int>(sizeof(T));
  }
  // Column of piece k's first element, relative to the segment.
  __device__ __forceinline__ int col(int k) const { return (lane + k * lanes) * N; }
  __device__ __forceinline__ bool has(int k) const { return k * lanes * N < left; }
  // Whether all elements of all pieces exist.
  __device__ __forceinline__ bool whole() const { return (kPieces - 1) * lanes * N + N <= left; }
  __device__ __forceinline__ int lead(const void* base, int64_t row, int64_t ld) const {
    return kShifted ? static_cast<int>(reinterpret_cast<uintptr_t>(static_cast<const T*>(base) + row * ld) & 15) : 0;
  }

  // Starts the copies of the warp's columns of a matrix's row into a slot.
  __device__ __forceinline__ void copy(uint32_t slot, const void* base, int64_t row, int64_t ld, int64_t rows, int64_t cols) const {
    const T* p = static_cast<const T*>(base) + row * ld + segment;
    if (!kShifted) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (has(k)) copy_async16(slot + static_cast<uint32_t>(lane + k * lanes) * 16u, p + col(k));
    } else {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = at & ~static_cast<uintptr_t>(15);
      const uintptr_t lo = reinterpret_cast<uintptr_t>(base), hi = lo + ((rows - 1) * ld + cols) * sizeof(T);
      const int bytes = static_cast<int>(at - first) + segment_bytes;
#pragma unroll
      for (int k = 0; k <= kPieces; ++k) {
        const int i = lane + k * lanes;
        if ((k == kPieces && lane > 0) || i * 16 >= bytes || segment_bytes == 0) continue;
        const uintptr_t w = first + static_cast<uintptr_t>(i) * 16;
        if (w >= lo && w + 16 <= hi) copy_async16(slot + static_cast<uint32_t>(i) * 16u, reinterpret_cast<const void*>(w));
        else copy_end(slot + static_cast<uint32_t>(i) * 16u, w, lo, hi);
      }
    }
  }
  // A word that reaches beyond the matrix's first or last element: the elements in it.
  static __device__ __noinline__ void copy_end(uint32_t slot, uintptr_t w, uintptr_t lo, uintptr_t hi) {
#pragma unroll 1
    for (int b = 0; b < 16; b += static_cast<int>(sizeof(T))) {
      if (w + b < lo || w + b >= hi) continue;
      if (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(slot + b), "r"(*reinterpret_cast<const uint32_t*>(w + b)) : "memory");
      else asm volatile("st.shared.u16 [%0], %1;" ::"r"(slot + b), "h"(*reinterpret_cast<const uint16_t*>(w + b)) : "memory");
    }
  }
  // Piece k of a row in a slot; 0 beyond the row.
  __device__ __forceinline__ void read(const uint8_t* slot, int lead, int k, bool in, float2 (&x)[W]) const {
    uint4 q = make_uint4(0, 0, 0, 0);
    const uint4* at = reinterpret_cast<const uint4*>(slot) + lane + k * lanes;
    if (in && has(k)) q = kShifted ? shifted<T>(at[0], at[1], lead) : at[0];
    Elem<T>::unpack(q, x);
    if (kShifted && !whole()) clip(k, x);
  }
  // Sets the elements beyond the row to zero.
  __device__ __forceinline__ void clip(int k, float2* x) const {
#pragma unroll
    for (int e = 0; e < W; ++e) {
      if (k * lanes * N + 2 * e >= left) x[e].x = 0.f;
      if (k * lanes * N + 2 * e + 1 >= left) x[e].y = 0.f;
    }
  }
  // Writes piece k of a row that starts at `row`, in order of k; `before` carries the piece before. All lanes of the warp call it.
  __device__ __forceinline__ void write(T* row, int k, const float2* x, bool in, uint4& before) const {
    const uint4 q = Elem<T>::pack(x);
    if (!kShifted) {
      if (in && has(k)) *reinterpret_cast<uint4*>(row + segment + col(k)) = q;
      return;
    }
    uint8_t* p = reinterpret_cast<uint8_t*>(row + segment);
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
    const bool last = lane == lanes - 1;
    const int from = static_cast<int>(threadIdx.x & 31) + (lane == 0 ? lanes - 1 : -1);
    uint4 prev;
    prev.x = __shfl_sync(kFull, last ? before.x : q.x, from);
    prev.y = __shfl_sync(kFull, last ? before.y : q.y, from);
    prev.z = __shfl_sync(kFull, last ? before.z : q.z, from);
    prev.w = __shfl_sync(kFull, last ? before.w : q.w, from);
    before = q;
    const int o = 16 * (lane + k * lanes) - lead;  // of the word, relative to the segment
    if (!in) return;
    const uint4 w = shifted<T>(prev, q, 16 - lead);
    if (o >= 0 && o + 16 <= segment_bytes) *reinterpret_cast<uint4*>(p + o) = w;
    else write_end(p, o, w);
    if (k == kPieces - 1 && last && lead > 0) write_end(p, o + 16, shifted<T>(q, make_uint4(0, 0, 0, 0), 16 - lead));
  }
  // The elements of a word that belong to the segment.
  __device__ __forceinline__ void write_end(uint8_t* p, int o, uint4 w) const {
    if (o + 16 <= 0 || o >= segment_bytes) return;
#pragma unroll 1
    for (int b = 0; b < 16; b += static_cast<int>(sizeof(T))) {
      const uint32_t bits = pop_front(w, T());
      if (o + b >= 0 && o + b < segment_bytes) *reinterpret_cast<typename Elem<T>::Bits*>(p + o + b) = static_cast<typename Elem<T>::Bits>(bits);
    }
  }
  // Column of element i (of 2 H), whether it exists, and a vector's elements there (`none` without a vector).
  __device__ __forceinline__ int element_col(int i) const { return segment + col(i / N) + i % N; }
  __device__ __forceinline__ bool has_element(int i) const { return i / N * lanes * N + i % N < left; }
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
#pragma unroll
    for (int i = 0; i < H; ++i) {
      x[i].x = has_element(2 * i) ? Elem<V>::get(v + element_col(2 * i)) : 0.f;
      x[i].y = has_element(2 * i + 1) ? Elem<V>::get(v + element_col(2 * i + 1)) : 0.f;
    }
  }
};

__device__ __forceinline__ void group_barrier(const RowShape& s, int group) {
  if (s.warps == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * s.warps) : "memory");
}

// Two sums over a row's threads, for each of them, in a fixed order. `turn`
// alternates between calls: a warp may be one call ahead of its group.
__device__ __forceinline__ float2 row_sum(float2 v, const RowShape& s, int group, int warp_in, Exchange& ex, int& turn) {
  for (int o = s.lanes >> 1; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(kFull, v.x, o);
    v.y += __shfl_xor_sync(kFull, v.y, o);
  }
  if (s.warps == 1) return v;
  float2* sum = ex.sum[turn] + group * s.warps;
  if ((threadIdx.x & 31) == 0) sum[warp_in] = v;
  group_barrier(s, group);
  v = sum[0];
  for (int w = 1; w < s.warps; ++w) v = add2(v, sum[w]);
  turn ^= 1;
  return v;
}

// Both rounded to T and widened again.
template <typename T>
__device__ __forceinline__ float2 round_pair(float2 x) {
  const T a = Elem<T>::make(x.x), b = Elem<T>::make(x.y);
  return make_float2(Elem<T>::get(&a), Elem<T>::get(&b));
}

// ------------------------------------------------------------------- host
constexpr int kMostPieces = 4;  // per thread

template <typename T>
bool starts_at_16(const void* p, int64_t ld) {
  return (reinterpret_cast<uintptr_t>(p) | (p ? ld * sizeof(T) : 0)) % 16 == 0;
}

// Lets a kernel have the ring's shared memory, once per device.
template <typename F>
cudaError_t allow_ring(F* kernel) {
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
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBudget);
    if (e != cudaSuccess) return e;
    bits |= uint64_t(1) << dev;
  }
  return cudaSuccess;
}

// Warps of a block, by the registers that a thread's elements leave.
inline int most_warps(int elements, bool heavy) {
  if (elements > 16) return heavy ? 12 : 16;
  return elements > 8 ? 20 : 32;
}

// How rows of `cols` elements, n of them to a piece, are shared out, with `matrices` copied per row. False: they
// are too long.
inline bool row_shape(int64_t cols, int n, bool shift, int matrices, bool heavy, RowShape* s, int* pieces) {
  const int64_t units = (cols + n - 1) / n;
  s->lanes = 32, s->warps = 1, *pieces = 1;
  if (units <= 16) {
    s->lanes = 1;
    while (s->lanes < units) s->lanes *= 2;
  } else {
    // Instructions per row: a warp's pieces, whether they exist or not, and about as many as one piece takes beside them.
    int64_t least = INT64_MAX;
    for (int k = kMostPieces; k >= 1; --k) {
      const int64_t warps = (units + 32 * k - 1) / (32 * k);
      if (warps > most_warps(n * k, heavy) || warps * (k + 1) >= least) continue;
      least = warps * (k + 1);
      s->warps = static_cast<int>(warps), *pieces = k;
    }
    if (least == INT64_MAX) return false;
  }
  s->groups = most_warps(n * *pieces, heavy) / s->warps;
  if (s->warps > 1 && s->groups > 15) s->groups = 15;  // named barriers
  s->slot_bytes = (s->lanes * *pieces + (shift ? 1 : 0)) * 16;
  auto fits = [&](int depth) { return static_cast<int64_t>(s->groups) * s->warps * (32 / s->lanes) * depth * matrices * s->slot_bytes <= kRingBudget; };
  while (s->groups > 1 && !fits(2)) --s->groups;
  if (!fits(2)) return false;
  s->depth = kMostDepth;
  while (!fits(s->depth)) --s->depth;
  return true;
}
inline int ring_bytes(const RowShape& s, int matrices) { return s.groups * s.warps * (32 / s.lanes) * s.depth * matrices * s.slot_bytes; }

// Shapes and launches, in files of their own. False: the rows are too long, nothing was launched.
bool launch_row_forward(const ForwardArgs& a, int type, int sms, cudaStream_t st, cudaError_t* e);
bool launch_row_backward(const BackwardArgs& a, int type, bool bias, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e);

}  // namespace norm
}  // namespace meq

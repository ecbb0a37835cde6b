// Rows of activations on their way through the norms' persistent kernels: how a
// row is shared out to threads, copied ahead into shared memory, and reduced.
//
// A group of `warps` warps takes a row at a time; of short rows a warp takes
// several at once, `lanes` lanes each. Column j of a row belongs to the same
// thread in every row, so weights stay in registers, and so do the sums over
// rows of the weight's gradient.
//
// Rows are copied into a ring of slots (cp.async) `depth` - 1 rows ahead, which
// keeps enough bytes on their way whatever the registers leave of the
// occupancy. Where every row starts at 16 bytes a thread copies the 16-byte
// pieces that it reads itself, and no thread waits for another. Else (kStep 1)
// the group copies the 16-byte words that hold the row, and each thread picks
// its elements out of them, wherever the row starts.
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
  int slot_bytes;  // of one matrix's row
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

// A thread's place in its row.
template <typename T, int kStep, int kPieces>
struct Place {
  static constexpr int E = kStep * kPieces, H = E / 2;  // elements of a thread, and pairs of them
  int cols, threads, t;  // threads of a row, and which of them this is
  int group, sub, warp_in;
  __device__ __forceinline__ Place(const RowShape& s, int64_t cols_) {
    const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
    cols = static_cast<int>(cols_);
    group = warp / s.warps;
    warp_in = warp - group * s.warps;
    sub = lane / s.lanes;
    threads = s.warps * s.lanes;
    t = warp_in * s.lanes + (lane - sub * s.lanes);
  }
  // Column of the thread's piece k.
  __device__ __forceinline__ int col(int k) const { return (t + k * threads) * kStep; }

  // Starts the copies of row `row` of a matrix into a slot. [lo, hi): the matrix's bytes.
  __device__ __forceinline__ void copy(uint32_t slot, const void* base, int64_t row, int64_t ld, int64_t rows) const {
    const T* p = static_cast<const T*>(base) + row * ld;
    if (kStep > 1) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (col(k) < cols) copy_async16(slot + static_cast<uint32_t>(t + k * threads) * 16u, p + col(k));
    } else {
      // Words that reach beyond the matrix's first or last element go element by element.
      const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = at & ~static_cast<uintptr_t>(15);
      const uintptr_t lo = reinterpret_cast<uintptr_t>(base), hi = lo + ((rows - 1) * ld + cols) * sizeof(T);
      const int words = static_cast<int>((at - first + cols * sizeof(T) + 15) / 16);
      for (int i = t; i < words; i += threads) {
        const uintptr_t w = first + static_cast<uintptr_t>(i) * 16;
        if (w >= lo && w + 16 <= hi) {
          copy_async16(slot + static_cast<uint32_t>(i) * 16u, reinterpret_cast<const void*>(w));
        } else {
#pragma unroll 1
          for (int b = 0; b < 16; b += static_cast<int>(sizeof(T))) {
            if (w + b < at || w + b >= at + cols * sizeof(T)) continue;
            const uint32_t d = slot + static_cast<uint32_t>(i) * 16u + b;
            if (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(d), "r"(*reinterpret_cast<const uint32_t*>(w + b)) : "memory");
            else asm volatile("st.shared.u16 [%0], %1;" ::"r"(d), "h"(*reinterpret_cast<const uint16_t*>(w + b)) : "memory");
          }
        }
      }
    }
  }
  // The thread's elements in units that lie together: pieces, or pairs of single elements.
  static constexpr int U = kStep > 1 ? kPieces : H, W = H / U;  // units, pairs of each
  // Where a row's elements start in its slot.
  __device__ __forceinline__ const uint8_t* row_at(const uint8_t* slot, const void* base, int64_t row, int64_t ld) const {
    return kStep > 1 ? slot : slot + (reinterpret_cast<uintptr_t>(static_cast<const T*>(base) + row * ld) & 15);
  }
  // Unit u of a row that lies in a slot; 0 beyond the row.
  __device__ __forceinline__ void read(const uint8_t* at, int u, bool in, float2 (&x)[W]) const {
    if (kStep > 1) {
      uint4 q = make_uint4(0, 0, 0, 0);
      if (in && col(u) < cols) q = reinterpret_cast<const uint4*>(at)[t + u * threads];
      Elem<T>::unpack(q, x);
    } else {
      const T* p = reinterpret_cast<const T*>(at);
      x[0].x = in && col(2 * u) < cols ? Elem<T>::get(p + col(2 * u)) : 0.f;
      x[0].y = in && col(2 * u + 1) < cols ? Elem<T>::get(p + col(2 * u + 1)) : 0.f;
    }
  }
  __device__ __forceinline__ void write(T* row, int u, const float2* x) const {
    if (kStep > 1) {
      if (col(u) < cols) *reinterpret_cast<uint4*>(row + col(u)) = Elem<T>::pack(x);
    } else {
      if (col(2 * u) < cols) row[col(2 * u)] = Elem<T>::make(x[0].x);
      if (col(2 * u + 1) < cols) row[col(2 * u + 1)] = Elem<T>::make(x[0].y);
    }
  }
  // Column of element i (of E), and a vector's elements there (`none` beyond the row).
  __device__ __forceinline__ int element_col(int i) const { return col(i / kStep) + i % kStep; }
  __device__ __forceinline__ void vector(const void* v, int type, float none, float2 (&x)[H]) const {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      x[i].x = v && element_col(2 * i) < cols ? load_as(v, type, element_col(2 * i)) : none;
      x[i].y = v && element_col(2 * i + 1) < cols ? load_as(v, type, element_col(2 * i + 1)) : none;
    }
  }
  // Sets the elements beyond the row to zero.
  __device__ __forceinline__ void clip(float2 (&x)[H]) const {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if (element_col(2 * i) >= cols) x[i].x = 0.f;
      if (element_col(2 * i + 1) >= cols) x[i].y = 0.f;
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
// Pieces (and single elements) per thread that the kernels are compiled for.
constexpr int kWholePieces[] = {1, 2, 3, 4}, kSingles[] = {2, 8, 16, 32};

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

// How rows of `cols` elements are shared out, `step` of them together, with `matrices` copied per row and
// at most `most` pieces per thread. pieces: per thread, as the kernels are compiled for. False: they are too long.
inline bool row_shape(int64_t cols, int step, int elem_size, int matrices, bool heavy, const int* compiled, int n_compiled, RowShape* s, int* pieces) {
  const int64_t units = (cols + step - 1) / step;
  s->lanes = 32, s->warps = 1;
  if (units <= 16 * compiled[0]) {
    *pieces = compiled[0];
    s->lanes = 1;
    while (static_cast<int64_t>(s->lanes) * compiled[0] < units) s->lanes *= 2;
  } else {
    const int most = compiled[n_compiled - 1];
    const int64_t warps = (units + 32 * most - 1) / (32 * most);
    if (warps > most_warps(step * most, heavy)) return false;
    s->warps = static_cast<int>(warps);
    const int64_t each = (units + 32 * warps - 1) / (32 * warps);
    for (int i = n_compiled - 1; i >= 0 && compiled[i] >= each; --i) *pieces = compiled[i];
  }
  s->groups = most_warps(step * *pieces, heavy) / s->warps;
  if (s->warps > 1 && s->groups > 15) s->groups = 15;  // named barriers
  s->slot_bytes = step > 1 ? s->warps * s->lanes * *pieces * 16 : static_cast<int>((cols * elem_size + 30) / 16 * 16);
  auto fits = [&](int depth) { return static_cast<int64_t>(s->groups) * (32 / s->lanes) * depth * matrices * s->slot_bytes <= kRingBudget; };
  while (s->groups > 1 && !fits(2)) --s->groups;
  if (!fits(2)) return false;
  s->depth = kMostDepth;
  while (!fits(s->depth)) --s->depth;
  return true;
}
inline int ring_bytes(const RowShape& s, int matrices) { return s.groups * (32 / s.lanes) * s.depth * matrices * s.slot_bytes; }

// Shapes and launches, in files of their own. False: the rows are too long, nothing was launched.
bool launch_row_forward(const ForwardArgs& a, int type, int sms, cudaStream_t st, cudaError_t* e);
bool launch_row_backward(const BackwardArgs& a, int type, bool bias, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e);

}  // namespace norm
}  // namespace meq

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

// Bytes `from` .. `from` + 15 of the 32 bytes of a and b (from: a multiple of the element's size, below 16).
template <typename T>
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int from) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
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
  __device__ __forceinline__ int lead(const void* base, uint32_t row, int64_t ld) const {
    return kShifted ? static_cast<int>((static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) + row * static_cast<uint32_t>(ld) * sizeof(T)) & 15) : 0;
  }

  // First element of a row, in a 32 x 64 bit product.
  static __device__ __forceinline__ uint64_t row_offset(uint32_t row, int64_t ld) { return static_cast<uint64_t>(row) * static_cast<uint64_t>(ld); }

  // Starts the copies of the warp's columns of a matrix's row into a slot.
  __device__ __forceinline__ void copy(uint32_t slot, const void* base, uint32_t row, int64_t ld, int64_t rows, int64_t cols) const {
    const T* p = static_cast<const T*>(base) + row_offset(row, ld) + segment;
    if (!kShifted) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (has(k)) copy_async16(slot + static_cast<uint32_t>(lane + k * lanes) * 16u, p + col(k));
    } else {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = at & ~static_cast<uintptr_t>(15);
      const uintptr_t lo = reinterpret_cast<uintptr_t>(base), hi = lo + ((rows - 1) * ld + cols) * sizeof(T);
      const int words = segment_bytes > 0 ? (static_cast<int>(at - first) + segment_bytes + 15) / 16 : 0;
      const bool inside = first >= lo && first + static_cast<uintptr_t>(words) * 16 <= hi;
      const uint32_t to = slot + static_cast<uint32_t>(lane) * 16u;
      const uintptr_t from = first + static_cast<uintptr_t>(lane) * 16;
#pragma unroll
      for (int k = 0; k <= kPieces; ++k) {
        if ((k == kPieces && lane > 0) || lane + k * lanes >= words) continue;
        if (inside) copy_async16(to + static_cast<uint32_t>(k * lanes) * 16u, reinterpret_cast<const void*>(from + k * lanes * 16));
        else copy_end(to + static_cast<uint32_t>(k * lanes) * 16u, from + k * lanes * 16, lo, hi);
      }
    }
  }
  // A word of a row whose words reach beyond the matrix's first or last element: the elements in it.
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
    if (kShifted && ends_in(k)) clip(k, x);
  }
  // Whether the row ends inside piece k.
  __device__ __forceinline__ bool ends_in(int k) const { return static_cast<unsigned>(left - k * lanes * N - 1) < static_cast<unsigned>(N - 1); }
  // Sets the elements beyond the row to zero.
  __device__ __forceinline__ void clip(int k, float2* x) const {
#pragma unroll
    for (int e = 0; e < W; ++e) {
      if (k * lanes * N + 2 * e >= left) x[e].x = 0.f;
      if (k * lanes * N + 2 * e + 1 >= left) x[e].y = 0.f;
    }
  }
  // The pieces of a row on their way to `row`, one after another: all lanes of the warp call write for each k in turn, then finish.
  struct Writer {
    uint8_t* p;    // the segment
    bool in;       // the row exists
    int lead;
    uint4 before;  // the piece before
    uint4 start, end;  // the words in which the segment starts and ends, where this lane holds them
    __device__ __forceinline__ Writer(T* row, const Place& place, bool in_) : p(reinterpret_cast<uint8_t*>(row + place.segment)), in(in_) {
      lead = kShifted ? static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15) : 0;
      before = start = end = make_uint4(0, 0, 0, 0);
    }
  };
  // The word in which the segment ends.
  __device__ __forceinline__ int end_word(int lead) const { return (segment_bytes + lead) / 16; }
  __device__ __forceinline__ void write(Writer& w, int k, const float2* x) const {
    const uint4 q = Elem<T>::pack(x);
    if (!kShifted) {
      if (w.in && has(k)) reinterpret_cast<uint4*>(w.p)[lane + k * lanes] = q;
      return;
    }
    const bool last = lane == lanes - 1;
    const int from = static_cast<int>(threadIdx.x & 31) + (lane == 0 ? lanes - 1 : -1), i = lane + k * lanes;
    uint4 prev;
    prev.x = __shfl_sync(kFull, last ? w.before.x : q.x, from);
    prev.y = __shfl_sync(kFull, last ? w.before.y : q.y, from);
    prev.z = __shfl_sync(kFull, last ? w.before.z : q.z, from);
    prev.w = __shfl_sync(kFull, last ? w.before.w : q.w, from);
    const uint4 word = w.lead ? shifted<T>(prev, q, 16 - w.lead) : q;
    w.before = q;
    if (i == end_word(w.lead)) w.end = word;
    if (i == 0) w.start = word;
    const int o = 16 * i - w.lead;  // of the word, relative to the segment
    if (w.in && o >= 0 && o + 16 <= segment_bytes) *reinterpret_cast<uint4*>(w.p + o) = word;
  }
  // The elements of the words in which the segment starts and ends, a lane each.
  __device__ __forceinline__ void finish(Writer& w) const {
    if (!kShifted) return;
    const int base = static_cast<int>(threadIdx.x & 31) & ~(lanes - 1), i = end_word(w.lead);
    // rows of one warp may start at different places: all lanes make both calls
    write_word(w, w.start, base, -w.lead, w.lead > 0);
    if (i == kPieces * lanes && lane == lanes - 1) w.end = shifted<T>(w.before, make_uint4(0, 0, 0, 0), (16 - w.lead) & 15);
    write_word(w, w.end, base + (i < kPieces * lanes ? i & (lanes - 1) : lanes - 1), 16 * i - w.lead, i > 0 || w.lead == 0);
  }
  // Those elements of lane `from`'s word, o bytes into the segment, that belong to the segment.
  __device__ __forceinline__ void write_word(const Writer& w, uint4 word, int from, int o, bool on) const {
    word.x = __shfl_sync(kFull, word.x, from);
    word.y = __shfl_sync(kFull, word.y, from);
    word.z = __shfl_sync(kFull, word.z, from);
    word.w = __shfl_sync(kFull, word.w, from);
#pragma unroll 1
    for (int e = lane; e < N; e += lanes) {
      const int b = o + e * static_cast<int>(sizeof(T));
      if (!w.in || !on || b < 0 || b >= segment_bytes) continue;
      const int at = e * static_cast<int>(sizeof(T)) / 4;
      const uint32_t pair = at & 2 ? (at & 1 ? word.w : word.z) : (at & 1 ? word.y : word.x);
      *reinterpret_cast<typename Elem<T>::Bits*>(w.p + b) = static_cast<typename Elem<T>::Bits>(sizeof(T) == 2 && (e & 1) ? pair >> 16 : pair);
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
    constexpr int kLoads = N / Elem<V>::N > 0 ? N / Elem<V>::N : 1;  // 16-byte loads per piece
    if (N >= Elem<V>::N && (reinterpret_cast<uintptr_t>(v) & 15) == 0) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
          uint4 q = make_uint4(0, 0, 0, 0);
          const int j = k * lanes * N + l * Elem<V>::N;
          float2* y = x + k * W + l * Elem<V>::N / 2;
          if (j + Elem<V>::N <= left) q = *reinterpret_cast<const uint4*>(v + segment + col(k) + l * Elem<V>::N);
          Elem<V>::unpack(q, y);
          if (j < left && j + Elem<V>::N > left) {
#pragma unroll
            for (int e = 0; e < Elem<V>::N; ++e)
              if (j + e < left) (e % 2 ? y[e / 2].y : y[e / 2].x) = Elem<V>::get(v + segment + col(k) + l * Elem<V>::N + e);
          }
        }
      }
      return;
    }
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
inline int most_warps(int elements) { return elements > 16 ? 16 : elements > 8 ? 20 : 32; }

// How rows of `cols` elements, n of them to a piece, are shared out, with `matrices` copied per row. False: they
// are too long.
inline bool row_shape(int64_t cols, int n, bool shift, int matrices, RowShape* s, int* pieces) {
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
      // shifting takes registers: four pieces of 16-bit elements spill 100 of them
      if (shift && n * k > 24 && units <= 32 * 3 * most_warps(n * 3)) continue;
      if (warps > most_warps(n * k) || warps * (k + 1) >= least) continue;
      least = warps * (k + 1);
      s->warps = static_cast<int>(warps), *pieces = k;
    }
    if (least == INT64_MAX) return false;
  }
  s->groups = most_warps(n * *pieces) / s->warps;
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

// Embedding lookup with scaling, and the gradient of its table.
//
//   out_i = scale E[t_i]                       (t_i < 0: zeros, t_i >= vocab: NaN)
//   dE[v] = scale sum over {i : t_i = v} of g_i   (+ what dE[v] held)
//
// HBM bounds both: a multiply or an addition per element moved.
//
// The gradient goes by sorted tokens, so every row of g is read once, every row
// of dE written once, and sums have a fixed order. Three launches:
//   sort_kernel    one cluster sorts the pairs (token, position) by token, stably,
//                  digit by digit, its counts exchanged through distributed shared
//                  memory; the other blocks meanwhile mark the tokens that occur
//                  and zero rows that do not, as many as the sort leaves time for
//   runs_kernel    a warp per chunk of 4 to 32 sorted pairs and slice of columns:
//                  runs of one token are summed and written; one that crosses the
//                  chunk's end is taken to its end if it is no longer than a chunk,
//                  else it leaves partial sums. Blocks between them zero the other
//                  rows, so that reads and writes share the memory's time.
//   joins_kernel   the partial sums of each long run, added in order
// Up to 256 tokens take one launch instead: a warp looks for its token's other
// occurrences among them itself.
#include <mutex>
#include <string>

#include "embedding_sort.cuh"
#include "meq_call.cuh"
#include "meq_elem.cuh"
#include "meq_elementwise.cuh"
#include "meq_mbar.cuh"

namespace meq {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr uint32_t kNoToken = 0xffffffffu;

// a / b in 32 bits where a fits: a division in 64 takes some 70 instructions, which were most of the lookup's.
__device__ __forceinline__ int64_t divide(int64_t a, int b) {
  if ((a >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}

// ------------------------------------------------------------------- lookup
struct LookupArgs {
  const int64_t* tokens;
  const void* table;
  void* out;
  int64_t n, vocab, cols, ld_table, ld_out;
  float scale;
};

// A lane's elements that lie together: 16 bytes of the result, since smaller stores cost more than what wider loads
// win (fp32 into bf16, 65536 x 2048: 71 us, with 8-byte stores and 16-byte loads instead of two 83).
template <typename Tout>
constexpr int kTogether = 16 / static_cast<int>(sizeof(Tout));
template <int kBytes>
struct Words;
struct Two {
  uint4 a, b;
};
template <>
struct Words<32> {
  using type = Two;
};
template <>
struct Words<16> {
  using type = uint4;
};
template <>
struct Words<8> {
  using type = uint2;
};
template <typename T, int kN>
using Piece = typename Words<kN * static_cast<int>(sizeof(T))>::type;

template <typename T>
__device__ __forceinline__ void widen(uint4 q, float2* x) {
  Elem<T>::unpack(q, x);
}
template <typename T>
__device__ __forceinline__ void widen(uint2 q, float2* x) {
  float2 y[4];
  Elem<T>::unpack(make_uint4(q.x, q.y, 0, 0), y);
  x[0] = y[0], x[1] = y[1];
}
template <typename T>
__device__ __forceinline__ void widen(Two q, float2* x) {
  Elem<T>::unpack(q.a, x);
  Elem<T>::unpack(q.b, x + 2);
}
template <typename W>
__device__ __forceinline__ W load_words(const W* p) {
  if constexpr (sizeof(W) == 32) return Two{__ldg(&p->a), __ldg(&p->b)};
  else return __ldg(p);
}

constexpr int kLookupThreads = 256, kLookupWarps = kLookupThreads / 32;
constexpr int kLookupCols = 512, kLookupFewCols = 128;  // of a warp, element by element: kPieces 0 and -1

// A warp takes a segment of 32 kPieces pieces of kTokens tokens' rows, or of shorter rows as many times 32 / lanes, `lanes`
// lanes each.
template <typename Tin, typename Tout, int kPieces, int kTokens>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const LookupArgs a, const int lanes, const int segments) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const float nan = __int_as_float(0x7fc00000);
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kLookupWarps + (threadIdx.x >> 5);
  const int lane = static_cast<int>(threadIdx.x & 31), sets = 32 / lanes;
  const int64_t group = divide(unit, segments), first = group * (sets * kTokens) + lane / lanes;
  if (first >= a.n) return;
  const int segment = static_cast<int>(unit - group * segments), cols = static_cast<int>(a.cols);
  int64_t t[kTokens];
#pragma unroll
  for (int u = 0; u < kTokens; ++u) t[u] = first + u * sets < a.n ? a.tokens[first + u * sets] : -1;
  auto known = [&](int u) { return t[u] >= 0 && t[u] < a.vocab; };
  auto row = [&](int u) { return static_cast<const Tin*>(a.table) + (known(u) ? t[u] : 0) * a.ld_table; };
  auto out = [&](int u) { return static_cast<Tout*>(a.out) + (first + u * sets) * a.ld_out; };
  auto none = [&](int u) { return t[u] < 0 ? 0.f : nan; };
  if constexpr (kPieces > 0) {
    constexpr int kN = kTogether<Tout>;
    const int j0 = (segment * kPieces * 32 + (lane & (lanes - 1))) * kN;
    Piece<Tin, kN> q[kTokens][kPieces];
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {  // every load, before the first store; those beyond the row read its start
        const int j = j0 + kN * lanes * k;
        q[u][k] = load_words(reinterpret_cast<const Piece<Tin, kN>*>(row(u) + (j < cols ? j : 0)));
      }
    }
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
      if (u > 0 && first + u * sets >= a.n) break;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int j = j0 + kN * lanes * k;
        float2 x[kN / 2];
        widen<Tin>(q[u][k], x);
#pragma unroll
        for (int e = 0; e < kN / 2; ++e) x[e] = known(u) ? mul2(x[e], make_float2(a.scale, a.scale)) : make_float2(none(u), none(u));
        if (j < cols) __stcs(reinterpret_cast<uint4*>(out(u) + j), Elem<Tout>::pack(x));
      }
    }
  } else {
    constexpr int kCols = kPieces == 0 ? kLookupCols : kLookupFewCols;
    const int j0 = segment * kCols + lane;
    typename Elem<Tin>::Bits q[kCols / 32];
#pragma unroll
    for (int k = 0; k < kCols / 32; ++k) q[k] = reinterpret_cast<const typename Elem<Tin>::Bits*>(row(0))[min(j0 + 32 * k, cols - 1)];
#pragma unroll
    for (int k = 0; k < kCols / 32; ++k) {
      const float x = Elem<Tin>::get(reinterpret_cast<const Tin*>(&q[k])) * a.scale;
      if (j0 + 32 * k < cols) out(0)[j0 + 32 * k] = Elem<Tout>::make(known(0) ? x : none(0));
    }
  }
}

// --------------------------------------------------------------------- sort
constexpr int kMostSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kRadixBits = 9, kRadix = 1 << kRadixBits;
constexpr int kSortKeys = 8;                    // groups of 32 keys that a warp has in registers
constexpr int kMarkWords = kSortWarps * kRadix; // of 32 rows each, that a block marks at a time

struct SortShared {
  uint32_t hist[kSortWarps][kRadix];  // counts, then next places, of each warp's keys; the other blocks: marks
  uint32_t total[kRadix];             // counts of the block
  uint32_t warp_sum[kSortWarps];
};

struct SortArgs {
  const int64_t* tokens;
  uint32_t n, vocab;
  uint32_t ctas;        // of the cluster that sorts
  int passes, bits;     // digits, and the bits of each
  uint2* pairs[2];      // the last pass writes pairs[0]
  uint32_t* crossing;   // the numbers of crossing runs: zeroed
  void* out;            // rows of tokens that do not occur are zeroed,
  int64_t row_bytes, ld_bytes;
  uint32_t words;       // 32 rows to a word of marks,
  uint32_t per_block;   // 2^32 / blocks that zero rows, rounded up: w blocks < 2^32 for every word w, so that __umulhi(w, it) = w / blocks
  uint32_t first_words; // those of the first words here,
  uint32_t* marks;      // the others by their marks, which are written here
};

__device__ __forceinline__ uint32_t key_of(int64_t t, uint32_t vocab) {
  return t >= 0 && t < static_cast<int64_t>(vocab) ? static_cast<uint32_t>(t) : vocab;  // tokens without a row go last
}

// Digit by digit from the lowest: a warp counts its consecutive keys' digits, the
// counts are summed over the warps of the block and the blocks of the cluster,
// and every key goes to its digit's next place, in the order of the keys. Lanes
// with the same digit find one another by a ballot per bit.
__device__ void sort_pairs(const SortArgs& a, SortShared& sh) {
  const uint32_t rank = blockIdx.x;
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const uint32_t per = (a.n + a.ctas * kSortWarps * 32 - 1) / (a.ctas * kSortWarps * 32) * 32;
  const uint64_t first64 = static_cast<uint64_t>(rank * kSortWarps + warp) * per;
  const uint32_t first = first64 < a.n ? static_cast<uint32_t>(first64) : a.n;
  const uint32_t last = a.n - first < per ? a.n : first + per;
  const uint32_t radix = 1u << a.bits, below = (1u << lane) - 1u;
  uint32_t* hist = sh.hist[warp];
  if (rank == 0 && threadIdx.x < 2) a.crossing[threadIdx.x] = 0;
  for (int p = 0; p < a.passes; ++p) {
    const uint2* src = a.pairs[(a.passes - p) & 1];
    uint2* dst = a.pairs[(a.passes - p - 1) & 1];
    const int shift = p * a.bits;
    uint2 pair[kSortKeys];
    uint32_t same[kSortKeys];  // lanes with the same digit (0: no key)
    auto load = [&](uint32_t base) {
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t i = base + 32 * k + lane;
        pair[k] = make_uint2(0, 0);
        if (i < last) pair[k] = p == 0 ? make_uint2(key_of(a.tokens[i], a.vocab), i) : __ldcg(src + i);
      }
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        same[k] = 0;
        if (base + 32 * k >= last) continue;
        const bool in = base + 32 * k + lane < last;
        const uint32_t key = pair[k].x >> shift;
        uint32_t m = __ballot_sync(kFull, in);
#pragma unroll
        for (int b = 0; b < kRadixBits; ++b) {
          if (b >= a.bits) break;
          const bool on = key & (1u << b);
          const uint32_t v = __ballot_sync(kFull, on);
          m &= v ^ (on ? 0u : kFull);
        }
        if (in) same[k] = m;
      }
    };
    auto digit = [&](int k) { return (pair[k].x >> shift) & (radix - 1); };
    for (uint32_t d = lane; d < radix; d += 32) hist[d] = 0;
    __syncwarp();
    for (uint32_t base = first; base < last; base += 32 * kSortKeys) {
      load(base);
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k)
        if (same[k] != 0 && (same[k] & below) == 0) atomicAdd(&hist[digit(k)], __popc(same[k]));
    }
    __syncthreads();
    const uint32_t d = threadIdx.x;
    if (d < radix) {
      uint32_t sum = 0;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) sum += sh.hist[w][d];
      sh.total[d] = sum;
    }
    cluster_sync_all();
    uint32_t all = 0, before = 0;
    if (d < radix) {
      uint32_t c[kMostSortCtas];
#pragma unroll
      for (uint32_t r = 0; r < kMostSortCtas; ++r) {
        c[r] = 0;
        if (r < a.ctas)
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[r]) : "r"(map_to_rank(smem_u32(&sh.total[d]), r)) : "memory");
      }
#pragma unroll
      for (uint32_t r = 0; r < kMostSortCtas; ++r) {
        before += r < rank ? c[r] : 0;
        all += c[r];
      }
    }
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(kFull, scan, o);
      if (lane >= o) scan += up;
    }
    if (lane == 31) sh.warp_sum[warp] = scan;
    __syncthreads();
    if (d < radix) {
      uint32_t at = scan - all + before;
      for (int w = 0; w < warp; ++w) at += sh.warp_sum[w];
#pragma unroll
      for (int w0 = 0; w0 < kSortWarps; w0 += 8) {
        uint32_t c[8];
#pragma unroll
        for (int w = 0; w < 8; ++w) c[w] = sh.hist[w0 + w][d];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          sh.hist[w0 + w][d] = at;
          at += c[w];
        }
      }
    }
    __syncthreads();
    for (uint32_t base = first; base < last; base += 32 * kSortKeys) {
      if (per > 32 * kSortKeys) load(base);  // else they are still there
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        if (base + 32 * k >= last) break;
        const uint32_t at = same[k] ? hist[digit(k)] : 0;
        __syncwarp();
        if (same[k]) {
          if ((same[k] & below) == 0) hist[digit(k)] = at + __popc(same[k]);
          dst[at + __popc(same[k] & below)] = pair[k];
        }
        __syncwarp();
      }
    }
    cluster_sync_all();  // the pairs are seen by the whole cluster, and nobody reads the totals any more
  }
}

// `threads` threads, of which this is the t-th, zero a row.
__device__ __forceinline__ void zero_row(uint8_t* p, int64_t bytes, int t, int threads) {
  const int64_t head = min(static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15), bytes);
  const int64_t pieces = (bytes - head) / 16, tail = head + 16 * pieces;
  for (int64_t i = t; i < pieces; i += threads) reinterpret_cast<uint4*>(p + head)[i] = make_uint4(0, 0, 0, 0);
  if (t < 8) {  // the ends: elements of 2 or 4 bytes
    const int64_t e = 2 * t;
    if (e < head) *reinterpret_cast<uint16_t*>(p + e) = 0;
    if (tail + e < bytes) *reinterpret_cast<uint16_t*>(p + tail + e) = 0;
  }
}

// Words of marks are dealt out to the blocks in turn: writes that advance through
// memory together run at 7 TB/s, those of a far-off share per SM at 5.
__device__ void zero_first_rows(const SortArgs& a, SortShared& sh) {
  uint32_t* marks = sh.hist[0];
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const uint32_t blocks = gridDim.x - a.ctas, block = blockIdx.x - a.ctas;
  for (uint32_t k0 = 0; block + blocks * static_cast<uint64_t>(k0) < a.words; k0 += kMarkWords) {
    const uint32_t here = min((a.words - block - blocks * k0 + blocks - 1) / blocks, static_cast<uint32_t>(kMarkWords));
    for (uint32_t i = threadIdx.x; i < here; i += kSortThreads) marks[i] = 0;
    __syncthreads();
    for (uint32_t base = 0; base < a.n; base += kSortThreads * kSortKeys) {
      int64_t t[kSortKeys];
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t i = base + k * kSortThreads + threadIdx.x;
        t[k] = i < a.n ? a.tokens[i] : -1;
      }
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t w = static_cast<uint32_t>(t[k]) >> 5, at = __umulhi(w, a.per_block);
        if (static_cast<uint64_t>(t[k]) < a.vocab && w - at * blocks == block && at - k0 < here) atomicOr(&marks[at - k0], 1u << (t[k] & 31));
      }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < here; i += kSortThreads)
      if (block + blocks * (k0 + i) >= a.first_words) a.marks[block + blocks * (k0 + i)] = marks[i];
    for (uint32_t i = 0; i < here && block + blocks * (k0 + i) < a.first_words; ++i) {
      const int64_t row = static_cast<int64_t>(block + blocks * (k0 + i)) * 32 + warp;
      if (row < a.vocab && !((marks[i] >> warp) & 1)) zero_row(static_cast<uint8_t*>(a.out) + row * a.ld_bytes, a.row_bytes, lane, 32);
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SortShared& sh = *reinterpret_cast<SortShared*>(smem_raw);
  pdl_allow_dependents();
  pdl_wait_predecessor();
  if (blockIdx.x < a.ctas) sort_pairs(a, sh);
  else zero_first_rows(a, sh);
}

// --------------------------------------------------------------------- runs
struct RunArgs {
  const void* grad;
  int64_t ld;
  uint32_t n, vocab;
  int cols, chunk;        // chunk: pairs of a chunk, 4 to 32
  const int64_t* tokens;  // few tokens
  const uint2* pairs;     // sorted ones
  uint32_t* crossing;     // [0], [1]: runs with partial sums in up to, and more than, kShortParts chunks more
  uint4* starts;          // the chunks in which they start, their tokens and the chunks more: `chunks` places for each of the two kinds
  uint32_t chunks;
  float* parts;           // [chunks][2][ld_parts]: sums of a run from the chunk before, of one into the next
  int64_t ld_parts;
  void* out;
  int64_t ld_out;
  int out_type, accumulate;
  float scale;
  // rows to zero: those of the words from first_word on, `fill_rows` per block, of `fills` blocks among the others
  int64_t row_bytes, ld_bytes;
  uint32_t first_word, fill_rows, fills, every;
  const uint32_t* marks;
};
constexpr int kRunThreads = 256, kRunWarps = kRunThreads / 32;
constexpr int kShortParts = 32;
constexpr uint32_t kFillBytes = 32768, kMostFillRows = 2048;  // of a block

// kN sums to consecutive elements of a row of the gradient; kN > 1: 16 bytes of floats, or as many elements of 16 bits, at a time.
template <int kN>
__device__ __forceinline__ void put(const RunArgs& a, int64_t i, const float (&sum)[kN]) {
  float old[kN] = {};
  if (a.out_type == MEQ_F32) {
    float* p = static_cast<float*>(a.out) + i;
    if constexpr (kN == 1) {
      if (a.accumulate) old[0] = *p;
      *p = fmaf(sum[0], a.scale, old[0]);
    } else {
      if (a.accumulate) {
#pragma unroll
        for (int e = 0; e < kN; e += 4) {
          const float4 q = *reinterpret_cast<const float4*>(p + e);
          old[e] = q.x, old[e + 1] = q.y, old[e + 2] = q.z, old[e + 3] = q.w;
        }
      }
#pragma unroll
      for (int e = 0; e < kN; e += 4)
        *reinterpret_cast<float4*>(p + e) = make_float4(fmaf(sum[e], a.scale, old[e]), fmaf(sum[e + 1], a.scale, old[e + 1]),
                                                        fmaf(sum[e + 2], a.scale, old[e + 2]), fmaf(sum[e + 3], a.scale, old[e + 3]));
    }
    return;
  }
  const bool bf = a.out_type == MEQ_BF16;
  uint16_t* p = static_cast<uint16_t*>(a.out) + i;
  auto widen = [&](uint32_t b) {
    return bf ? __uint_as_float(b << 16) : __half2float(__ushort_as_half(static_cast<uint16_t>(b)));
  };
  auto narrow = [&](float x) -> uint32_t {
    return bf ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
  };
  if constexpr (kN == 1) {
    if (a.accumulate) old[0] = widen(*p);
    *p = static_cast<uint16_t>(narrow(fmaf(sum[0], a.scale, old[0])));
  } else {
    uint32_t w[kN / 2];
    if (a.accumulate) {
#pragma unroll
      for (int e = 0; e < kN; e += 4) {
        const uint2 q = *reinterpret_cast<const uint2*>(p + e);
        old[e] = widen(q.x & 0xFFFFu), old[e + 1] = widen(q.x >> 16), old[e + 2] = widen(q.y & 0xFFFFu), old[e + 3] = widen(q.y >> 16);
      }
    }
#pragma unroll
    for (int e = 0; e < kN; e += 2)
      w[e / 2] = narrow(fmaf(sum[e], a.scale, old[e])) | narrow(fmaf(sum[e + 1], a.scale, old[e + 1])) << 16;
    if constexpr (kN == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

// A lane's columns of a slice, and their sums. kStep: columns that lie together (a 16-byte piece, or one element).
template <typename T, int kStep, int kPieces>
struct Slice {
  static constexpr int kCols = 32 * kStep * kPieces;
  int j0, cols;
  float acc[kPieces][kStep];
  __device__ __forceinline__ Slice(int slice, int lane, int cols_) : j0(slice * kCols + lane * kStep), cols(cols_) { clear(); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
      for (int i = 0; i < kStep; ++i) acc[k][i] = 0.f;
  }
  __device__ __forceinline__ int col(int k) const { return j0 + 32 * kStep * k; }
  struct Row {
    uint4 q[kStep > 1 ? kPieces : 1];
    typename Elem<T>::Bits s[kStep > 1 ? 1 : kPieces];
  };
  // Single elements (kStep 1), kAhead rows of them at a time. Unconditional, so that the loads of several rows are on their
  // way together: columns beyond the row read its start.
  static constexpr int kAhead = 4;
  __device__ __forceinline__ void load(Row& r, const T* row) const {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) r.s[k] = reinterpret_cast<const typename Elem<T>::Bits*>(row)[col(k) < cols ? col(k) : 0];
  }
  __device__ __forceinline__ void add(const Row& r) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if constexpr (kStep == 1) {
        acc[k][0] += Elem<T>::get(reinterpret_cast<const T*>(&r.s[k]));
      } else {
        float2 x[kStep / 2];
        Elem<T>::unpack(r.q[k], x);
#pragma unroll
        for (int i = 0; i < kStep / 2; ++i) {
          const float2 sum = add2(make_float2(acc[k][2 * i], acc[k][2 * i + 1]), x[i]);
          acc[k][2 * i] = sum.x, acc[k][2 * i + 1] = sum.y;
        }
      }
    }
  }
  // Rows in a ring of a warp's shared memory, each lane its own pieces (kStep > 1).
  static constexpr int kSlots = kStep > 1 ? 16 / kPieces : 1, kRingBytes = kStep > 1 ? kSlots * kPieces * 512 : 0;
  static constexpr int kFewSlots = kStep > 1 ? kSlots / 2 : 1;  // where blocks that zero rows have the same shared memory
  __device__ __forceinline__ void copy(uint32_t ring, int slot, const T* row) const {
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + static_cast<uint32_t>((slot * kPieces + k) * 512)),
                   "l"(row + (col(k) < cols ? col(k) : 0))
                   : "memory");
  }
  __device__ __forceinline__ void take(Row& r, const uint4* ring, int slot) const {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) r.q[k] = ring[(slot * kPieces + k) * 32];
  }
  __device__ __forceinline__ void finish(const RunArgs& a, uint32_t token) const {
    const int64_t row = static_cast<int64_t>(token) * a.ld_out;
    if constexpr (kStep == 1) {  // what the row holds is on its way for all columns before the first is written
      float old[kPieces] = {};
      if (a.accumulate) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
          if (col(k) < cols) old[k] = held(a, row + col(k));
      }
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (col(k) < cols) set(a, row + col(k), fmaf(acc[k][0], a.scale, old[k]));
    } else {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (col(k) < cols) put(a, row + col(k), acc[k]);
    }
  }
  static __device__ __forceinline__ float held(const RunArgs& a, int64_t i) {
    if (a.out_type == MEQ_F32) return static_cast<const float*>(a.out)[i];
    if (a.out_type == MEQ_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.out)[i]);
    return __half2float(static_cast<const __half*>(a.out)[i]);
  }
  static __device__ __forceinline__ void set(const RunArgs& a, int64_t i, float x) {
    if (a.out_type == MEQ_F32) static_cast<float*>(a.out)[i] = x;
    else if (a.out_type == MEQ_BF16) static_cast<__nv_bfloat16*>(a.out)[i] = __float2bfloat16_rn(x);
    else static_cast<__half*>(a.out)[i] = __float2half_rn(x);
  }
  __device__ __forceinline__ void leave(float* part) const {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if (col(k) >= cols) continue;
      if constexpr (kStep == 1) {
        part[col(k)] = acc[k][0];
      } else {
#pragma unroll
        for (int i = 0; i < kStep; i += 4)
          *reinterpret_cast<float4*>(part + col(k) + i) = make_float4(acc[k][i], acc[k][i + 1], acc[k][i + 2], acc[k][i + 3]);
      }
    }
  }
};

// Whether this block zeroes rows, and its number among those that do, or among the others. Of the two kinds the one with
// fewer blocks has every a.every-th block of the grid, as long as they last.
__device__ __forceinline__ bool fill_block(const RunArgs& a, int64_t* index) {
  const uint32_t fewer = min(a.fills, gridDim.x - a.fills), at = blockIdx.x / a.every;
  const bool few = at < fewer && at * a.every == blockIdx.x;
  *index = few ? at : blockIdx.x - min(fewer, at + 1);
  return few == (a.fills <= gridDim.x - a.fills);
}
// Zeroes this block's rows but those marked(row, number in the block).
template <typename F>
__device__ __forceinline__ void fill_rows(const RunArgs& a, int64_t block, F marked) {
  const int64_t row0 = static_cast<int64_t>(a.first_word) * 32 + block * a.fill_rows;
  const int rows = static_cast<int>(min(static_cast<int64_t>(a.fill_rows), static_cast<int64_t>(a.vocab) - row0));
  const int threads = a.fill_rows >= kRunWarps ? 32 : kRunThreads;  // of a row
  for (int r = static_cast<int>(threadIdx.x) / threads; r < rows; r += kRunThreads / threads)
    if (!marked(row0 + r, r))
      zero_row(static_cast<uint8_t*>(a.out) + (row0 + r) * a.ld_bytes, a.row_bytes, static_cast<int>(threadIdx.x) % threads, threads);
}

template <typename T, int kStep, int kPieces>
__global__ void __launch_bounds__(kRunThreads, kStep > 1 ? 4 : 3) runs_kernel(const __grid_constant__ RunArgs a) {
  using S = Slice<T, kStep, kPieces>;
  pdl_allow_dependents();
  pdl_wait_predecessor();
  int64_t block;
  if (fill_block(a, &block)) {
    fill_rows(a, block, [&](int64_t row, int) { return (a.marks[row >> 5] >> (row & 31)) & 1; });
    return;
  }
  const int lane = static_cast<int>(threadIdx.x & 31);
  const int slices = (a.cols + S::kCols - 1) / S::kCols;
  const int64_t unit = block * kRunWarps + (threadIdx.x >> 5), c = divide(unit, slices), first = c * a.chunk;
  if (first >= a.n) return;
  auto pair_at = [&](int64_t i) { return i >= 0 && i < a.n ? a.pairs[i] : make_uint2(kNoToken, 0); };
  const uint2 pair = lane < a.chunk ? pair_at(first + lane) : make_uint2(kNoToken, 0);
  const uint2 next = pair_at(first + a.chunk + lane), prev = pair_at(first - 1 - lane);
  auto ones = [](uint32_t m) { return m == kFull ? 32 : __ffs(~m) - 1; };  // from the lowest bit on
  const int count = __popc(__ballot_sync(kFull, pair.x < a.vocab));  // the others come last
  if (count == 0) return;
  // The runs at the chunk's ends: how far they reach beyond it (32 or more: 32), and whether one is taken whole by the chunk
  // in which it starts.
  const uint32_t key0 = __shfl_sync(kFull, pair.x, 0), key1 = __shfl_sync(kFull, pair.x, count - 1);
  const int back = ones(__ballot_sync(kFull, prev.x == key0)), lead = __popc(__ballot_sync(kFull, pair.x == key0));
  const int ahead = count == a.chunk ? ones(__ballot_sync(kFull, next.x == key1)) : 0, tail = __popc(__ballot_sync(kFull, pair.x == key1));
  const bool through = lead == a.chunk;  // one run from end to end
  const bool skip = back > 0 && back + lead + (through ? ahead : 0) <= a.chunk;
  const bool take = ahead > 0 && !(through && back > 0) && tail + ahead <= a.chunk;
  const int begin = skip ? lead : 0, end = count + (take ? ahead : 0);
  const int part_end = back > 0 && !skip ? lead - 1 : -1;  // last pair of a run from before
  const bool into_next = ahead > 0 && !take && !(through && back > 0);
  S s(static_cast<int>(unit - c * slices), lane, a.cols);
  const T* grad = static_cast<const T*>(a.grad);
  auto key = [&](int e) { return e < a.chunk ? __shfl_sync(kFull, pair.x, e) : __shfl_sync(kFull, next.x, e - a.chunk); };
  auto row_of = [&](int e) {
    const uint32_t pos = e < a.chunk ? __shfl_sync(kFull, pair.y, e & 31) : __shfl_sync(kFull, next.y, (e - a.chunk) & 31);
    return grad + static_cast<int64_t>(pos) * a.ld;
  };
  uint32_t now = key(begin);
  // After pair e: its run's sum, if it ends here.
  auto end_run = [&](int e) {
    const uint32_t k = now;
    if (e + 1 < end) {
      now = key(e + 1);
      if (now == k) return;
    }
    if (e == part_end) {
      s.leave(a.parts + 2 * c * a.ld_parts);
    } else if (e == end - 1 && into_next) {
      s.leave(a.parts + (2 * c + 1) * a.ld_parts);
      if (s.j0 < 32 * kStep) {  // the first slice's warp
        // the chunks after this one that begin with the token: their partial sums belong to it
        uint32_t more = 0;
        for (int n = 32; n == 32; more += n) {
          const int64_t i = first + (more + 1 + lane) * static_cast<int64_t>(a.chunk);
          n = ones(__ballot_sync(kFull, i < a.n && a.pairs[i].x == k));
        }
        if (lane == 0) {
          const int longer = more > kShortParts;
          a.starts[longer * a.chunks + atomicAdd(&a.crossing[longer], 1u)] = make_uint4(static_cast<uint32_t>(c), k, more, 0);
        }
      }
    } else {
      s.finish(a, k);
    }
    s.clear();
  };
  if constexpr (kStep > 1) {
    extern __shared__ __align__(16) uint8_t ring_raw[];
    uint4* ring = reinterpret_cast<uint4*>(ring_raw + (threadIdx.x >> 5) * S::kRingBytes) + lane;
    const uint32_t ring32 = smem_u32(ring);
#pragma unroll 1
    for (int u = 0; u < S::kSlots - 1; ++u) {
      if (begin + u < end) s.copy(ring32, u, row_of(begin + u));
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    int slot = 0;
#pragma unroll 1
    for (int e = begin; e < end; ++e) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kSlots - 2) : "memory");
      typename S::Row r;
      s.take(r, ring, slot);
      s.add(r);
      const int put = slot == 0 ? S::kSlots - 1 : slot - 1;  // the slot of the row before
      if (e + S::kSlots - 1 < end) s.copy(ring32, put, row_of(e + S::kSlots - 1));
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++slot == S::kSlots) slot = 0;
      end_run(e);
    }
  } else {
    constexpr int kAhead = S::kAhead;
#pragma unroll 1
    for (int e0 = begin; e0 < end; e0 += kAhead) {
      typename S::Row r[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) s.load(r[u], row_of(min(e0 + u, end - 1)));
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (e0 + u >= end) break;
        s.add(r[u]);
        end_run(e0 + u);
      }
    }
  }
}

// Few tokens, unsorted: a warp per token and slice of columns takes its token's rows if none precedes it, in order. One
// launch for three: 256 tokens into 32000 x 768 fp32 16.2 us, 257, sorted, 21.8; added to 3000 x 768 3.4 and 13.8. The
// price is one token many times over, which one warp adds up: 256 times the same 43 us, 257 times 9.9.
template <typename T, int kStep, int kPieces>
__global__ void __launch_bounds__(kRunThreads) few_kernel(const __grid_constant__ RunArgs a) {
  using S = Slice<T, kStep, kPieces>;
  __shared__ uint32_t marks[kMostFillRows / 32];
  __shared__ int64_t tokens[kFewTokens];
  pdl_allow_dependents();
  pdl_wait_predecessor();
  int64_t block;
  if (fill_block(a, &block)) {
    for (int i = static_cast<int>(threadIdx.x); i < static_cast<int>(kMostFillRows / 32); i += kRunThreads) marks[i] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.n; i += kRunThreads) {
      const int64_t at = a.tokens[i] - block * a.fill_rows;
      if (at >= 0 && at < a.fill_rows) atomicOr(&marks[at >> 5], 1u << (at & 31));
    }
    __syncthreads();
    fill_rows(a, block, [&](int64_t, int r) { return (marks[r >> 5] >> (r & 31)) & 1; });
    return;
  }
  for (uint32_t i = threadIdx.x; i < kFewTokens; i += kRunThreads) tokens[i] = i < a.n ? a.tokens[i] : -1;
  __syncthreads();
  const int lane = static_cast<int>(threadIdx.x & 31), n = static_cast<int>(a.n);
  const int slices = (a.cols + S::kCols - 1) / S::kCols;
  const int64_t unit = block * kRunWarps + (threadIdx.x >> 5);
  const int i = static_cast<int>(divide(unit, slices));
  if (i >= n) return;
  const int64_t token = tokens[i];
  if (token < 0 || token >= a.vocab) return;
  for (int q = 0; 32 * q < i; ++q)
    if (__ballot_sync(kFull, 32 * q + lane < i && tokens[32 * q + lane] == token)) return;
  int q = i / 32;
  uint32_t hits = __ballot_sync(kFull, 32 * q + lane >= i && tokens[32 * q + lane] == token);
  auto next = [&]() {  // position of the token's next occurrence, -1: no more
    while (hits == 0 && 32 * (q + 1) < n) {
      ++q;
      hits = __ballot_sync(kFull, tokens[32 * q + lane] == token);
    }
    const int at = hits ? 32 * q + __ffs(hits) - 1 : -1;
    hits &= hits - 1;
    return at;
  };
  S s(static_cast<int>(unit - static_cast<int64_t>(i) * slices), lane, a.cols);
  auto row_of = [&](int at) { return static_cast<const T*>(a.grad) + static_cast<int64_t>(at) * a.ld; };
  if constexpr (kStep > 1) {
    extern __shared__ __align__(16) uint8_t ring_raw[];
    uint4* ring = reinterpret_cast<uint4*>(ring_raw + (threadIdx.x >> 5) * S::kRingBytes / 2) + lane;
    const uint32_t ring32 = smem_u32(ring);
    int copied = 0, slot = 0;
#pragma unroll 1
    for (int u = 0; u < S::kFewSlots - 1; ++u) {
      const int at = next();
      if (at >= 0) s.copy(ring32, u, row_of(at)), ++copied;
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
#pragma unroll 1
    for (int taken = 0; taken < copied; ++taken) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kFewSlots - 2) : "memory");
      typename S::Row r;
      s.take(r, ring, slot);
      s.add(r);
      const int at = next();
      if (at >= 0) s.copy(ring32, slot == 0 ? S::kFewSlots - 1 : slot - 1, row_of(at)), ++copied;
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++slot == S::kFewSlots) slot = 0;
    }
  } else {
    constexpr int kAhead = S::kAhead;
#pragma unroll 1
    for (int rows = kAhead; rows == kAhead;) {
      typename S::Row r[kAhead];
      rows = 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = next();
        s.load(r[u], row_of(at < 0 ? i : at));
        rows += at >= 0;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (u < rows) s.add(r[u]);
    }
  }
  s.finish(a, static_cast<uint32_t>(token));
}

// The runs with partial sums. Of up to kShortParts chunks, a block takes 1024 columns, 128 of them a warp; of more, a block
// takes 128 columns and deals the partial sums out to its warps.
constexpr int kJoinCols = 128;
__global__ void __launch_bounds__(kRunThreads) joins_kernel(const __grid_constant__ RunArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ float4 sh[kRunWarps][32];
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const int64_t narrow = (a.cols + kJoinCols - 1) / kJoinCols, wide = (narrow + kRunWarps - 1) / kRunWarps;
  const int64_t longs = narrow * a.crossing[1], units = longs + wide * a.crossing[0];
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const bool is_long = u < longs;
    const int64_t v = is_long ? u : u - longs, per = is_long ? narrow : wide, run = divide(v, static_cast<int>(per));
    const uint4 start = a.starts[(is_long ? a.chunks : 0) + run];
    const int64_t c = start.x, more = start.z;
    const uint32_t token = start.y;
    const int j = static_cast<int>(is_long ? v - run * per : (v - run * per) * kRunWarps + warp) * kJoinCols + 4 * lane;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* part = a.parts + j;
    if (j < a.cols) {
      if (!is_long || warp == 0) s = *reinterpret_cast<const float4*>(part + (2 * c + 1) * a.ld_parts);
#pragma unroll 8
      for (int64_t k = is_long ? 1 + warp : 1; k <= more; k += is_long ? kRunWarps : 1) {
        const float4 x = *reinterpret_cast<const float4*>(part + 2 * (c + k) * a.ld_parts);
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
    }
    if (is_long) {
      __syncthreads();  // sh is free
      sh[warp][lane] = s;
      __syncthreads();
      if (warp != 0) continue;
#pragma unroll
      for (int w = 1; w < kRunWarps; ++w) {
        const float4 x = sh[w][lane];
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
    }
    const float sum[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < a.cols) {
        const float one[1] = {sum[e]};
        put(a, static_cast<int64_t>(token) * a.ld_out + j + e, one);
      }
  }
}

// --------------------------------------------------------------------- host
// A grid of `units` shared out to blocks of `per`.
cudaError_t grid_of(int64_t units, int64_t per, dim3* grid) {
  const int64_t blocks = (units + per - 1) / per;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  *grid = dim3(static_cast<unsigned>(blocks));
  return cudaSuccess;
}

template <typename Tin, typename Tout>
cudaError_t launch_lookup(const LookupArgs& a, cudaStream_t st) {
  constexpr int kN = kTogether<Tout>, kMost = kN * sizeof(Tin) == 32 ? 2 : 4;
  const size_t in = kN * sizeof(Tin) > 16 ? 16 : kN * sizeof(Tin);
  const bool pieces = a.cols % kN == 0 && a.ld_table % kN == 0 && a.ld_out % kN == 0 && aligned_to(a.table, in) && aligned_to(a.out, 16);
  // A warp has kMost pieces per lane under way: of one token, or where a token needs fewer of two or four.
  int lanes = 32, each = 1, segments = 1;
  auto* kernel = lookup_kernel<Tin, Tout, kMost, 1>;
  if (pieces) {
    while (lanes > 1 && a.cols / kN <= lanes / 2) lanes /= 2;
    const int64_t need = (a.cols / kN + 31) / 32;
    if (need == 1) kernel = lookup_kernel<Tin, Tout, 1, kMost>, each = kMost;
    else if (need == 2 && kMost == 4) kernel = lookup_kernel<Tin, Tout, 2, 2>, each = 2;
    else segments = static_cast<int>((need + kMost - 1) / kMost);
  } else {
    const bool narrow = a.cols <= kLookupFewCols;
    kernel = narrow ? lookup_kernel<Tin, Tout, -1, 1> : lookup_kernel<Tin, Tout, 0, 1>;
    segments = narrow ? 1 : static_cast<int>((a.cols + kLookupCols - 1) / kLookupCols);
  }
  const int64_t tokens = 32 / lanes * each;
  dim3 grid;
  const cudaError_t e = grid_of((a.n + tokens - 1) / tokens * segments, kLookupWarps, &grid);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, grid, dim3(kLookupThreads), 0, st, 1, a, lanes, segments);
}
template <typename Tin>
cudaError_t launch_lookup(const LookupArgs& a, int out_type, cudaStream_t st) {
  if (out_type == MEQ_F32) return launch_lookup<Tin, float>(a, st);
  if (out_type == MEQ_BF16) return launch_lookup<Tin, __nv_bfloat16>(a, st);
  return launch_lookup<Tin, __half>(a, st);
}

// Rows are zeroed beside the sort for as long as it takes, at the rate here; the others beside the sums. At 0, 1.5, 3, 4.5
// and 6 TB/s, us: 65536 tokens into 151936 x 4096 bf16 290, 286, 282, 282, 284, 8192 into 32000 x 768 fp32 37, 35, 33, 32, 31.
constexpr double kSortUs = 9.0, kSortUsPerToken = 0.0002, kFillBytesPerUs = 4.5e6;

// Pairs of a chunk: fewer where few tokens would leave warps without work (6000 x 1001 accumulating 28 us, from 1216 units
// on 36; larger calls within 5% from 1216 to 9728).
int chunk_for(int64_t n, int64_t cols) {
  int chunk = 32;
  while (chunk > 4 && (n + chunk - 1) / chunk * ((cols + 255) / 256) < 4864) chunk /= 2;
  return chunk;
}
struct Work {
  int64_t pairs0, pairs1, starts, crossing, marks, parts, floats;  // offsets in floats
  int64_t chunks, ld_parts;
};
Work work_for(int64_t n, int64_t vocab, int64_t cols) {
  Work w{};
  if (n <= kFewTokens) return w;
  w.chunks = (n + chunk_for(n, cols) - 1) / chunk_for(n, cols);
  w.ld_parts = (cols + 3) / 4 * 4;
  w.pairs1 = 2 * n;
  w.starts = (4 * n + 3) / 4 * 4;
  w.crossing = w.starts + 8 * w.chunks;
  w.marks = w.crossing + 2;
  w.parts = (w.marks + (vocab + 31) / 32 + 3) / 4 * 4;
  w.floats = w.parts + 2 * w.chunks * w.ld_parts;
  return w;
}

// Clusters of 8 or 16 blocks of the sort that the device holds at a time (0: none), asked once per device.
cudaError_t prepared_sort(int ctas, int* clusters) {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static int known[kMaxDevices][2] = {};  // and one more, 0: not asked yet
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  int& most = known[dev][ctas == 16];
  if (most == 0) {
    e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(SortShared)));
    if (e == cudaSuccess && ctas == 16) e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = sizeof(SortShared);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(ctas);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, sort_kernel, &cfg);
    if (e != cudaSuccess) return e;
    most = 1 + (n > 0 ? n : 0);
  }
  *clusters = most - 1;
  return cudaSuccess;
}

template <typename T, int kStep, int kPieces>
cudaError_t launch_runs(RunArgs a, cudaStream_t st) {
  constexpr int kCols = Slice<T, kStep, kPieces>::kCols;
  const bool few = a.n <= kFewTokens;
  dim3 grid;
  const int64_t slices = (a.cols + kCols - 1) / kCols;
  const cudaError_t e = grid_of((few ? a.n : a.chunks) * slices + static_cast<int64_t>(a.fills) * kRunWarps, kRunWarps, &grid);
  if (e != cudaSuccess) return e;
  const uint32_t others = grid.x - a.fills, fewer = others < a.fills ? others : a.fills;
  a.every = fewer > 0 ? grid.x / fewer : grid.x;
  constexpr int kRing = kRunWarps * Slice<T, kStep, kPieces>::kRingBytes;
  auto* kernel = few ? few_kernel<T, kStep, kPieces> : runs_kernel<T, kStep, kPieces>;
  const cudaError_t ready = allow_shared(kernel, kRing);
  if (ready != cudaSuccess) return ready;
  return launch_pdl(kernel, grid, dim3(kRunThreads), few ? kRing / 2 : kRing, st, 1, a);
}
template <typename T>
cudaError_t launch_runs_of(const RunArgs& a, cudaStream_t st) {
  constexpr int kN = Elem<T>::N;
  const size_t out = static_cast<size_t>(kN) * elem_bytes(a.out_type) < 16 ? 8 : 16;
  const bool whole = a.cols % kN == 0 && a.ld % kN == 0 && aligned_to(a.grad, 16) && aligned_to(a.out, out) &&
                     a.ld_out * elem_bytes(a.out_type) % out == 0;
  if (!whole) return launch_runs<T, 1, 8>(a, st);
  return a.cols / kN > 32 ? launch_runs<T, kN, 2>(a, st) : launch_runs<T, kN, 1>(a, st);
}

}  // namespace
}  // namespace meq

using namespace meq;

extern "C" {

meq_status meq_embedding(const int64_t* tokens, int64_t n, const void* table, int table_type, int64_t vocab, int64_t cols, int64_t ld_table,
                         float scale, void* out, int out_type, int64_t ld_out, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why;
    if (!valid_type(table_type) || !valid_type(out_type)) why = "the types must be meq_dtypes";
    else if (n < 0 || n > (int64_t(1) << 27)) why = "n must be in 0..2^27";
    else if (vocab < 1 || vocab > (int64_t(1) << 28)) why = "vocab must be in 1..2^28";
    else if (cols < 1 || cols > (int64_t(1) << 20)) why = "cols must be in 1..2^20";
    else if ((vocab > 1 && ld_table < cols) || (n > 1 && ld_out < cols)) why = "the row strides must be at least cols";
    else if (ld_table < 0 || ld_table > (int64_t(1) << 34) || ld_out < 0 || ld_out > (int64_t(1) << 34)) why = "the row strides must be in 0..2^34";
    else if (n > 0 && (!tokens || !table || !out)) why = "tokens, table and out must not be NULL";
    else if (!aligned_to(tokens, 8) || !aligned_to(table, elem_bytes(table_type)) || !aligned_to(out, elem_bytes(out_type)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_embedding: " + why);
    if (n == 0) return MEQ_OK;
    const LookupArgs a{tokens, table, out, n, vocab, cols, ld_table, ld_out, scale};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = table_type == MEQ_F32    ? launch_lookup<float>(a, out_type, st)
                          : table_type == MEQ_BF16 ? launch_lookup<__nv_bfloat16>(a, out_type, st)
                                                   : launch_lookup<__half>(a, out_type, st);
    return launch_status(e, "meq_embedding", "launch");
  });
}

int64_t meq_embedding_work_floats(int64_t n, int64_t vocab, int64_t cols) {
  return n < 0 || vocab < 1 || cols < 1 ? 0 : work_for(n, vocab, cols).floats + 4;
}

meq_status meq_embedding_grad(const void* grad, int type, int64_t n, int64_t cols, int64_t ld, const int64_t* tokens, int64_t vocab,
                              float scale, void* out, int out_type, int64_t ld_out, int accumulate, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why;
    if (!valid_type(type) || !valid_type(out_type)) why = "the types must be meq_dtypes";
    else if (n < 0 || n > (int64_t(1) << 27)) why = "n must be in 0..2^27";
    else if (vocab < 1 || vocab > (int64_t(1) << 28)) why = "vocab must be in 1..2^28";
    else if (cols < 1 || cols > (int64_t(1) << 20)) why = "cols must be in 1..2^20";
    else if ((n > 1 && ld < cols) || (vocab > 1 && ld_out < cols)) why = "the row strides must be at least cols";
    else if (ld < 0 || ld > (int64_t(1) << 34) || ld_out < 0 || ld_out > (int64_t(1) << 34)) why = "the row strides must be in 0..2^34";
    else if (!out || (n > 0 && (!grad || !tokens))) why = "grad, tokens and out must not be NULL";
    else if (!work || !aligned_to(work, 16)) why = "work must not be NULL and be 16-byte aligned";
    else if (!aligned_to(tokens, 8) || !aligned_to(grad, elem_bytes(type)) || !aligned_to(out, elem_bytes(out_type)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_embedding_grad: " + why);
    if (n == 0 && accumulate) return MEQ_OK;
    cudaError_t e = cudaSuccess;
    int clusters = 0, sms = 0;
    auto clusters_of = [&](int blocks) {
      if (e != cudaSuccess) cudaGetLastError();  // 16 blocks are not to be had, which 8 make good
      int held = 0;
      e = prepared_sort(blocks, &held);
      return held;
    };
    const int ctas = sort_blocks(n, clusters_of, &clusters);
    if (ctas > 0 && e == cudaSuccess && clusters < 1) e = cudaErrorInvalidConfiguration;
    if (ctas > 0 && e == cudaSuccess) sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_embedding_grad", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Work w = work_for(n, vocab, cols);
    RunArgs a{};
    a.grad = grad, a.ld = ld, a.n = static_cast<uint32_t>(n), a.vocab = static_cast<uint32_t>(vocab), a.cols = static_cast<int>(cols);
    a.out = out, a.ld_out = ld_out, a.out_type = out_type, a.accumulate = accumulate != 0, a.scale = scale;
    a.row_bytes = cols * elem_bytes(out_type), a.ld_bytes = ld_out * elem_bytes(out_type);
    if (!accumulate) {
      a.fill_rows = static_cast<uint32_t>(a.row_bytes >= kFillBytes ? 1 : kFillBytes / a.row_bytes);
      if (a.fill_rows > kMostFillRows) a.fill_rows = kMostFillRows;
    }
    if (ctas > 0) {
      SortArgs s{};
      s.tokens = tokens, s.n = a.n, s.vocab = a.vocab;
      int bits = 1;  // of the largest key, vocab
      while (bits < 32 && (vocab >> bits) != 0) ++bits;
      s.passes = (bits + kRadixBits - 1) / kRadixBits;
      s.bits = (bits + s.passes - 1) / s.passes;
      s.pairs[0] = reinterpret_cast<uint2*>(work + w.pairs0), s.pairs[1] = reinterpret_cast<uint2*>(work + w.pairs1);
      s.crossing = reinterpret_cast<uint32_t*>(work + w.crossing);
      s.ctas = static_cast<uint32_t>(ctas);
      if (accumulate) clusters = 1;
      else if (clusters < 2) clusters = 2;
      if (!accumulate) {
        s.out = out, s.row_bytes = a.row_bytes, s.ld_bytes = a.ld_bytes;
        s.words = static_cast<uint32_t>((vocab + 31) / 32);
        const uint64_t fill = static_cast<uint64_t>((clusters - 1) * ctas);
        s.per_block = static_cast<uint32_t>(((uint64_t(1) << 32) + fill - 1) / fill);
        // what can be written while the tokens are sorted
        const double bytes = (kSortUs + kSortUsPerToken * static_cast<double>(n)) * kFillBytesPerUs;
        const double words = bytes / (32.0 * static_cast<double>(a.row_bytes));
        s.first_words = words < s.words ? static_cast<uint32_t>(words) : s.words;
        s.marks = reinterpret_cast<uint32_t*>(work + w.marks);
        a.first_word = s.first_words, a.marks = s.marks;
      }
      e = launch_pdl(sort_kernel, dim3(static_cast<unsigned>(clusters * ctas)), dim3(kSortThreads), sizeof(SortShared), st, ctas, s);
      if (e != cudaSuccess) return launch_status(e, "meq_embedding_grad", "sort launch");
      a.pairs = s.pairs[0], a.crossing = s.crossing, a.starts = reinterpret_cast<uint4*>(work + w.starts);
      a.chunk = chunk_for(n, cols), a.chunks = static_cast<uint32_t>(w.chunks);
      a.parts = work + w.parts, a.ld_parts = w.ld_parts;
    } else {
      a.tokens = tokens;
    }
    const int64_t rest = vocab - static_cast<int64_t>(a.first_word) * 32;
    if (!accumulate && rest > 0) a.fills = static_cast<uint32_t>((rest + a.fill_rows - 1) / a.fill_rows);
    e = type == MEQ_F32 ? launch_runs_of<float>(a, st) : type == MEQ_BF16 ? launch_runs_of<__nv_bfloat16>(a, st) : launch_runs_of<__half>(a, st);
    if (e != cudaSuccess || ctas == 0) return launch_status(e, "meq_embedding_grad", "sum launch");
    const int64_t most = w.chunks * ((cols + 8 * kJoinCols - 1) / (8 * kJoinCols)), blocks = 2 * static_cast<int64_t>(sms);
    e = launch_pdl(joins_kernel, dim3(static_cast<unsigned>(most < blocks ? most : blocks)), dim3(kRunThreads), 0, st, 1, a);
    return launch_status(e, "meq_embedding_grad", "join launch");
  });
}

}  // extern "C"

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
//                  in their share of the vocabulary, and zero the other rows
//   runs_kernel    a warp per chunk of 4 to 32 sorted pairs and slice of columns:
//                  runs of one token inside the chunk are summed and written, runs
//                  that cross its ends leave a partial sum
//   joins_kernel   the partial sums of each crossing run, added in order
#include <mutex>
#include <string>

#include "meq_call.cuh"
#include "meq_elem.cuh"
#include "meq_elementwise.cuh"
#include "meq_mbar.cuh"

namespace meq {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr uint32_t kNoToken = 0xffffffffu;

// ------------------------------------------------------------------- lookup
struct LookupArgs {
  const int64_t* tokens;
  const void* table;
  void* out;
  int64_t n, vocab, cols, ld_table, ld_out;
  float scale;
};

// Eight consecutive elements, 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float2 (&x)[4]) {
  const uint4* q = reinterpret_cast<const uint4*>(p);
  Elem<T>::unpack(__ldg(q), x);
  if (Elem<T>::N == 4) Elem<T>::unpack(__ldg(q + 1), x + 2);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float2 (&x)[4]) {
  uint4* q = reinterpret_cast<uint4*>(p);
  __stcs(q, Elem<T>::pack(x));
  if (Elem<T>::N == 4) __stcs(q + 1, Elem<T>::pack(x + 2));
}

constexpr int kLookupThreads = 256;
constexpr int kLookupPieces = 4;   // of eight elements, per thread
constexpr int kLookupCols = 512;   // of a warp, element by element

template <typename Tin, typename Tout, bool kPieces>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const LookupArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const float nan = __int_as_float(0x7fc00000);
  if (kPieces) {
    const uint32_t per_row = static_cast<uint32_t>(a.cols / 8);
    const int64_t total = a.n * per_row;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (kLookupThreads * kLookupPieces) + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kLookupPieces; ++k) {
      const int64_t at = first + k * kLookupThreads;
      if (at >= total) break;
      const int64_t i = at / per_row;
      const int64_t j = (at - i * per_row) * 8;
      const int64_t t = a.tokens[i];
      float2 x[4];
      if (t >= 0 && t < a.vocab) {
        load8(static_cast<const Tin*>(a.table) + t * a.ld_table + j, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = mul2(x[e], make_float2(a.scale, a.scale));
      } else {
        const float v = t < 0 ? 0.f : nan;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = make_float2(v, v);
      }
      store8(static_cast<Tout*>(a.out) + i * a.ld_out + j, x);
    }
  } else {
    const int64_t segments = (a.cols + kLookupCols - 1) / kLookupCols;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kLookupThreads / 32) + (threadIdx.x >> 5);
    const int64_t i = unit / segments;
    if (i >= a.n) return;
    const int64_t j0 = (unit - i * segments) * kLookupCols + (threadIdx.x & 31);
    const int64_t t = a.tokens[i];
    const bool known = t >= 0 && t < a.vocab;
    const Tin* row = static_cast<const Tin*>(a.table) + (known ? t : 0) * a.ld_table;
    Tout* out = static_cast<Tout*>(a.out) + i * a.ld_out;
#pragma unroll
    for (int k = 0; k < kLookupCols / 32; ++k) {
      const int64_t j = j0 + 32 * k;
      if (j < a.cols) out[j] = Elem<Tout>::make(known ? Elem<Tin>::get(row + j) * a.scale : t < 0 ? 0.f : nan);
    }
  }
}

// --------------------------------------------------------------------- sort
constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kRadixBits = 9, kRadix = 1 << kRadixBits;
constexpr int kSortKeys = 8;      // groups of 32 keys that a warp loads ahead
constexpr int kMarkBits = kSortWarps * kRadix * 32;  // rows that a block's marks cover at a time

struct SortShared {
  uint32_t hist[kSortWarps][kRadix];  // counts, then next places, of each warp's keys; the other blocks: marks
  uint32_t total[kRadix];             // counts of the block
  uint32_t warp_sum[kSortWarps];
};

struct SortArgs {
  const int64_t* tokens;
  uint32_t n, vocab;
  int passes, bits;     // digits, and the bits of each
  uint2* pairs[2];      // the last pass writes pairs[0]
  uint32_t* crossing;   // the number of crossing runs: zeroed
  void* out;            // rows of tokens that do not occur are zeroed; NULL: left
  int64_t row_bytes, ld_bytes;
};

__device__ __forceinline__ uint32_t key_of(int64_t t, uint32_t vocab) {
  return t >= 0 && t < static_cast<int64_t>(vocab) ? static_cast<uint32_t>(t) : vocab;  // tokens without a row go last
}

// Digit by digit from the lowest: a warp counts its consecutive keys' digits, the
// counts are summed over the warps of the block and the blocks of the cluster,
// and every key goes to its digit's next place, in the order of the keys.
__device__ void sort_pairs(const SortArgs& a, SortShared& sh) {
  const uint32_t rank = blockIdx.x;
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const uint32_t per = (a.n + kSortCtas * kSortWarps * 32 - 1) / (kSortCtas * kSortWarps * 32) * 32;
  const uint64_t first64 = static_cast<uint64_t>(rank * kSortWarps + warp) * per;
  const uint32_t first = first64 < a.n ? static_cast<uint32_t>(first64) : a.n;
  const uint32_t last = a.n - first < per ? a.n : first + per;
  const uint32_t radix = 1u << a.bits, below = (1u << lane) - 1u;
  uint32_t* hist = sh.hist[warp];
  if (rank == 0 && threadIdx.x == 0) *a.crossing = 0;
  for (int p = 0; p < a.passes; ++p) {
    const uint2* src = a.pairs[(a.passes - p) & 1];
    uint2* dst = a.pairs[(a.passes - p - 1) & 1];
    const int shift = p * a.bits;
    auto load = [&](uint32_t i) -> uint2 {
      if (p == 0) return make_uint2(key_of(a.tokens[i], a.vocab), i);
      return __ldcg(src + i);
    };
    for (uint32_t d = lane; d < radix; d += 32) hist[d] = 0;
    __syncwarp();
    for (uint32_t base = first; base < last; base += 32 * kSortKeys) {
      uint32_t key[kSortKeys];
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t i = base + 32 * k + lane;
        key[k] = i < last ? load(i).x : 0;
      }
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const bool in = base + 32 * k + lane < last;
        const uint32_t d = in ? (key[k] >> shift) & (radix - 1) : radix;
        const uint32_t same = __match_any_sync(kFull, d);
        if (in && (same & below) == 0) hist[d] += __popc(same);
        __syncwarp();
      }
    }
    __syncthreads();
    const uint32_t d = threadIdx.x;
    if (d < radix) {
      uint32_t sum = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = sh.hist[w][d];
        sh.hist[w][d] = sum;
        sum += c;
      }
      sh.total[d] = sum;
    }
    cluster_sync_all();
    uint32_t all = 0, before = 0;
    if (d < radix)
      for (uint32_t r = 0; r < kSortCtas; ++r) {
        uint32_t c;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(map_to_rank(smem_u32(&sh.total[d]), r)) : "memory");
        before += r < rank ? c : 0;
        all += c;
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
      for (int w = 0; w < kSortWarps; ++w) sh.hist[w][d] += at;
    }
    __syncthreads();
    for (uint32_t base = first; base < last; base += 32 * kSortKeys) {
      uint2 pair[kSortKeys];
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t i = base + 32 * k + lane;
        pair[k] = i < last ? load(i) : make_uint2(0, 0);
      }
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const bool in = base + 32 * k + lane < last;
        const uint32_t digit = in ? (pair[k].x >> shift) & (radix - 1) : radix;
        const uint32_t same = __match_any_sync(kFull, digit);
        const uint32_t at = in ? hist[digit] : 0;
        __syncwarp();
        if (in) {
          if ((same & below) == 0) hist[digit] = at + __popc(same);
          dst[at + __popc(same & below)] = pair[k];
        }
        __syncwarp();
      }
    }
    cluster_sync_all();  // the pairs are seen by the whole cluster, and nobody reads the totals any more
  }
}

__device__ __forceinline__ void zero_row(uint8_t* p, int64_t bytes, int lane) {
  const int64_t head = min(static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15), bytes);
  const int64_t pieces = (bytes - head) / 16, tail = head + 16 * pieces;
  for (int64_t i = lane; i < pieces; i += 32) __stcs(reinterpret_cast<uint4*>(p + head) + i, make_uint4(0, 0, 0, 0));
  // the ends: elements of 2 or 4 bytes
  const int64_t e = 2 * lane;
  if (e < head) *reinterpret_cast<uint16_t*>(p + e) = 0;
  if (tail + e < bytes) *reinterpret_cast<uint16_t*>(p + tail + e) = 0;
}

__device__ void zero_other_rows(const SortArgs& a, SortShared& sh) {
  uint32_t* marks = sh.hist[0];
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const int64_t blocks = gridDim.x - kSortCtas, block = blockIdx.x - kSortCtas;
  const int64_t share = (a.vocab + blocks - 1) / blocks, end = min((block + 1) * share, static_cast<int64_t>(a.vocab));
  for (int64_t v0 = block * share; v0 < end; v0 += kMarkBits) {
    const int64_t rows = min(end - v0, static_cast<int64_t>(kMarkBits));
    for (int64_t i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) marks[i] = 0;
    __syncthreads();
    for (uint32_t base = 0; base < a.n; base += kSortThreads * kSortKeys) {
      int64_t t[kSortKeys];
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k) {
        const uint32_t i = base + k * kSortThreads + threadIdx.x;
        t[k] = i < a.n ? a.tokens[i] : -1;
      }
#pragma unroll
      for (int k = 0; k < kSortKeys; ++k)
        if (t[k] >= v0 && t[k] < v0 + rows) atomicOr(&marks[(t[k] - v0) >> 5], 1u << ((t[k] - v0) & 31));
    }
    __syncthreads();
    for (int64_t i = warp; i < rows; i += kSortWarps)
      if (((marks[i >> 5] >> (i & 31)) & 1u) == 0) zero_row(static_cast<uint8_t*>(a.out) + (v0 + i) * a.ld_bytes, a.row_bytes, lane);
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SortShared& sh = *reinterpret_cast<SortShared*>(smem_raw);
  pdl_allow_dependents();
  pdl_wait_predecessor();
  if (blockIdx.x < kSortCtas) sort_pairs(a, sh);
  else zero_other_rows(a, sh);
}

// --------------------------------------------------------------------- runs
struct RunArgs {
  const void* grad;
  int64_t ld;
  uint32_t n, vocab;
  int cols, chunk;       // chunk: pairs of a chunk, 4 to 32
  const uint2* pairs;
  uint32_t* crossing;    // [0]: number of crossing runs, then the chunks in which they start
  float* parts;          // [chunks][2][ld_parts]: sums of a run from the chunk before, of one into the next
  int64_t ld_parts;
  void* out;
  int64_t ld_out;
  int out_type, accumulate;
  float scale;
};
constexpr int kRunThreads = 256;

__device__ __forceinline__ void put(void* out, int type, int64_t i, float sum, float scale, int accumulate) {
  if (type == MEQ_F32) {
    float* p = static_cast<float*>(out) + i;
    *p = accumulate ? fmaf(sum, scale, *p) : sum * scale;
  } else if (type == MEQ_BF16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(out) + i;
    *p = __float2bfloat16_rn(accumulate ? fmaf(sum, scale, __bfloat162float(*p)) : sum * scale);
  } else {
    __half* p = static_cast<__half*>(out) + i;
    *p = __float2half_rn(accumulate ? fmaf(sum, scale, __half2float(*p)) : sum * scale);
  }
}

// kStep: columns that lie together in a lane (a 16-byte piece, or one element); kPieces: of those per lane.
template <typename T, int kStep, int kPieces>
__global__ void __launch_bounds__(kRunThreads) runs_kernel(const RunArgs a) {
  constexpr int kAhead = kStep == 1 ? 2 : (8 / kPieces > 4 ? 4 : 8 / kPieces);  // rows loaded ahead
  pdl_allow_dependents();
  const int lane = static_cast<int>(threadIdx.x & 31);
  const int slices = (a.cols + 32 * kStep * kPieces - 1) / (32 * kStep * kPieces);
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kRunThreads / 32) + (threadIdx.x >> 5);
  const int64_t c = unit / slices;
  const int j0 = static_cast<int>(unit - c * slices) * (32 * kStep * kPieces) + lane * kStep;  // + 32 kStep k
  pdl_wait_predecessor();
  const int64_t first = c * a.chunk;
  if (first >= a.n) return;
  auto key_at = [&](int64_t i) { return i >= 0 && i < a.n ? a.pairs[i].x : kNoToken; };
  uint2 pair = make_uint2(kNoToken, 0);
  if (lane < a.chunk && first + lane < a.n) pair = a.pairs[first + lane];
  const int count = __popc(__ballot_sync(kFull, pair.x < a.vocab));  // the others come last
  if (count == 0) return;
  const uint32_t before = key_at(first - 1), after = key_at(first + a.chunk);
  const T* grad = static_cast<const T*>(a.grad);
  float acc[kPieces * kStep];
#pragma unroll
  for (int k = 0; k < kPieces * kStep; ++k) acc[k] = 0.f;
  bool from_before = __shfl_sync(kFull, pair.x, 0) == before;
  for (int e0 = 0; e0 < count; e0 += kAhead) {
    uint4 q[kAhead][kPieces];
    float s[kAhead][kPieces];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t pos = __shfl_sync(kFull, pair.y, (e0 + u) & 31);
      const T* row = grad + static_cast<int64_t>(pos) * a.ld;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int j = j0 + 32 * kStep * k;
        const bool in = e0 + u < count && j < a.cols;
        if (kStep == 1) s[u][k] = in ? Elem<T>::get(row + j) : 0.f;
        else q[u][k] = in ? __ldcs(reinterpret_cast<const uint4*>(row + j)) : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int e = e0 + u;
      if (e >= count) break;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        if (kStep == 1) {
          acc[k] += s[u][k];
        } else {
          float2 x[kStep / 2 + 1];
          Elem<T>::unpack(q[u][k], x);
#pragma unroll
          for (int i = 0; i < kStep / 2; ++i) acc[k * kStep + 2 * i] += x[i].x, acc[k * kStep + 2 * i + 1] += x[i].y;
        }
      }
      const uint32_t key = __shfl_sync(kFull, pair.x, e);
      const uint32_t next = e + 1 < a.chunk ? __shfl_sync(kFull, pair.x, (e + 1) & 31) : after;
      if (next == key && e + 1 < a.chunk) continue;
      // the run's end in this chunk
      const bool into_next = next == key;
      if (!from_before && !into_next) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          const int j = j0 + 32 * kStep * k;
          if (j < a.cols) {
#pragma unroll
            for (int i = 0; i < kStep; ++i)
              put(a.out, a.out_type, static_cast<int64_t>(key) * a.ld_out + j + i, acc[k * kStep + i], a.scale, a.accumulate);
          }
        }
      } else {
        float* part = a.parts + (2 * c + (from_before ? 0 : 1)) * a.ld_parts;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          const int j = j0 + 32 * kStep * k;
          if (j < a.cols) {
#pragma unroll
            for (int i = 0; i < kStep; ++i) part[j + i] = acc[k * kStep + i];
          }
        }
        if (!from_before && j0 == 0) a.crossing[1 + atomicAdd(a.crossing, 1u)] = static_cast<uint32_t>(c);
      }
      from_before = false;
#pragma unroll
      for (int k = 0; k < kPieces * kStep; ++k) acc[k] = 0.f;
    }
  }
}

// The crossing runs: a block per run and 128 columns, the run's partial sums dealt out to its warps.
constexpr int kJoinCols = 128;
__global__ void __launch_bounds__(kRunThreads) joins_kernel(const RunArgs a) {
  constexpr int kWarps = kRunThreads / 32;
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ float4 sh[kWarps][32];
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  const int64_t slices = (a.cols + kJoinCols - 1) / kJoinCols, units = slices * *a.crossing;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t c = a.crossing[1 + u / slices];
    const int j = static_cast<int>(u % slices) * kJoinCols + 4 * lane;
    const uint32_t token = a.pairs[c * a.chunk + a.chunk - 1].x;
    int64_t more = 0;  // chunks after c that begin with the token
    for (;;) {
      const int64_t i = (c + 1 + more + lane) * a.chunk;
      const uint32_t others = __ballot_sync(kFull, i >= a.n || a.pairs[i].x != token);
      if (others) {
        more += __ffs(others) - 1;
        break;
      }
      more += 32;
    }
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j < a.cols) {
#pragma unroll 4
      for (int64_t k = warp; k <= more; k += kWarps) {
        const float4 x = *reinterpret_cast<const float4*>(a.parts + (2 * (c + k) + (k == 0 ? 1 : 0)) * a.ld_parts + j);
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < kWarps; ++w) {
        const float4 x = sh[w][lane];
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
      const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < a.cols) put(a.out, a.out_type, static_cast<int64_t>(token) * a.ld_out + j + i, v[i], a.scale, a.accumulate);
    }
    __syncthreads();
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
  constexpr size_t kIn = 16 / sizeof(Tin), kOut = 16 / sizeof(Tout);
  const bool pieces = a.cols % 8 == 0 && a.ld_table % kIn == 0 && a.ld_out % kOut == 0 && aligned_to(a.table, 16) && aligned_to(a.out, 16);
  dim3 grid;
  const cudaError_t e = pieces ? grid_of(a.n * (a.cols / 8), kLookupThreads * kLookupPieces, &grid)
                               : grid_of(a.n * ((a.cols + kLookupCols - 1) / kLookupCols), kLookupThreads / 32, &grid);
  if (e != cudaSuccess) return e;
  return launch_pdl(pieces ? lookup_kernel<Tin, Tout, true> : lookup_kernel<Tin, Tout, false>, grid, dim3(kLookupThreads), 0, st, 1, a);
}
template <typename Tin>
cudaError_t launch_lookup(const LookupArgs& a, int out_type, cudaStream_t st) {
  if (out_type == MEQ_F32) return launch_lookup<Tin, float>(a, st);
  if (out_type == MEQ_BF16) return launch_lookup<Tin, __nv_bfloat16>(a, st);
  return launch_lookup<Tin, __half>(a, st);
}

// Pairs of a chunk: fewer where few tokens would leave warps without work.
int chunk_for(int64_t n, int64_t cols) {
  int chunk = 32;
  while (chunk > 4 && (n + chunk - 1) / chunk * ((cols + 255) / 256) < 2432) chunk /= 2;
  return chunk;
}
struct Work {
  int64_t pairs0, pairs1, crossing, parts, floats;  // offsets in floats
  int64_t chunks, ld_parts;
};
Work work_for(int64_t n, int64_t cols) {
  Work w;
  w.chunks = (n + chunk_for(n, cols) - 1) / chunk_for(n, cols);
  w.ld_parts = (cols + 3) / 4 * 4;
  w.pairs0 = 0;
  w.pairs1 = 2 * n;
  w.crossing = 4 * n;
  w.parts = (w.crossing + 1 + w.chunks + 3) / 4 * 4;
  w.floats = w.parts + 2 * w.chunks * w.ld_parts;
  return w;
}

cudaError_t prepared_sort() {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static bool known[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[dev]) {
    e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(SortShared)));
    if (e != cudaSuccess) return e;
    known[dev] = true;
  }
  return cudaSuccess;
}

template <typename T, int kStep, int kPieces>
cudaError_t launch_runs(const RunArgs& a, int64_t chunks, cudaStream_t st) {
  dim3 grid;
  const cudaError_t e = grid_of(chunks * ((a.cols + 32 * kStep * kPieces - 1) / (32 * kStep * kPieces)), kRunThreads / 32, &grid);
  if (e != cudaSuccess) return e;
  return launch_pdl(runs_kernel<T, kStep, kPieces>, grid, dim3(kRunThreads), 0, st, 1, a);
}
template <typename T>
cudaError_t launch_runs_of(const RunArgs& a, int64_t chunks, cudaStream_t st) {
  constexpr int kN = Elem<T>::N;
  if (a.cols % kN != 0 || a.ld % kN != 0 || !aligned_to(a.grad, 16)) return launch_runs<T, 1, 16>(a, chunks, st);
  const int pieces = a.cols / kN;
  if (pieces > 64) return launch_runs<T, kN, 4>(a, chunks, st);
  if (pieces > 32) return launch_runs<T, kN, 2>(a, chunks, st);
  return launch_runs<T, kN, 1>(a, chunks, st);
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

int64_t meq_embedding_work_floats(int64_t n, int64_t cols) { return n < 0 || cols < 1 ? 0 : work_for(n, cols).floats; }

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
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e == cudaSuccess) e = prepared_sort();
    if (e != cudaSuccess) return launch_status(e, "meq_embedding_grad", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Work w = work_for(n, cols);
    SortArgs s{};
    s.tokens = tokens, s.n = static_cast<uint32_t>(n), s.vocab = static_cast<uint32_t>(vocab);
    int bits = 1;  // of the largest key, vocab
    while (bits < 32 && (vocab >> bits) != 0) ++bits;
    s.passes = (bits + kRadixBits - 1) / kRadixBits;
    s.bits = (bits + s.passes - 1) / s.passes;
    s.pairs[0] = reinterpret_cast<uint2*>(work + w.pairs0), s.pairs[1] = reinterpret_cast<uint2*>(work + w.pairs1);
    s.crossing = reinterpret_cast<uint32_t*>(work + w.crossing);
    s.out = out, s.row_bytes = cols * elem_bytes(out_type), s.ld_bytes = ld_out * elem_bytes(out_type);
    const int fill = accumulate ? 0 : (sms + kSortCtas - 1) / kSortCtas * kSortCtas - kSortCtas;
    e = launch_pdl(sort_kernel, dim3(static_cast<unsigned>(kSortCtas + fill)), dim3(kSortThreads), sizeof(SortShared), st, kSortCtas, s);
    if (e != cudaSuccess) return launch_status(e, "meq_embedding_grad", "sort launch");
    if (n == 0) return MEQ_OK;
    RunArgs a{};
    a.grad = grad, a.ld = ld, a.n = s.n, a.vocab = s.vocab, a.cols = static_cast<int>(cols), a.chunk = chunk_for(n, cols);
    a.pairs = s.pairs[0], a.crossing = s.crossing, a.parts = work + w.parts, a.ld_parts = w.ld_parts;
    a.out = out, a.ld_out = ld_out, a.out_type = out_type, a.accumulate = accumulate != 0, a.scale = scale;
    e = type == MEQ_F32 ? launch_runs_of<float>(a, w.chunks, st) : type == MEQ_BF16 ? launch_runs_of<__nv_bfloat16>(a, w.chunks, st) : launch_runs_of<__half>(a, w.chunks, st);
    if (e != cudaSuccess) return launch_status(e, "meq_embedding_grad", "sum launch");
    e = launch_pdl(joins_kernel, dim3(static_cast<unsigned>(2 * sms)), dim3(kRunThreads), 0, st, 1, a);
    return launch_status(e, "meq_embedding_grad", "join launch");
  });
}

}  // extern "C"

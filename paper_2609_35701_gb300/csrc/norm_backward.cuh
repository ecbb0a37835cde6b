// The backward pass of the norms: rows that the registers of a group of warps
// hold. One persistent block per SM; dy and h are read once, dx written once, and
// the sums over rows of dy xhat and dy stay in registers until the block's last
// row; then the block's groups are added up and leave one partial sum per column.
//
// Bound by HBM where rows are long and many, us (at the copy rate): RMS norm
// 32768 x 4096 bf16 with dh 157 (161). Layer norms of long rows by latency: of 32
// elements a thread an SM holds 16 warps, which issue in 0.53 of its slots (670
// instructions per warp and row of 1024 columns; RMS norm with dh 540, 0.39) and
// else wait for loads and for their group's barriers: 16384 x 4096 77 (60), 16384 x
// 8192 161 (121), where an SM has two groups of eight warps and rings of two rows.
// Rows off 16 bytes alike: 16384 x 2047 67 (30). Small ones by the launch, the first
// load, the groups' sums and the second launch: 8192 x 1024 17.5 (7.5), of which 5
// come after the last row.
//
// Few rows (kFew): one cluster of at most eight blocks, which reads the partial
// sums in its shared memory and writes the sums themselves, without a second
// launch. Its kernels are compiled apart: with both endings in one, the rows'
// registers spilled and 8192 x 1024 fp16 took 18.9 us for 17.2.
#pragma once
#include "norm_rows.cuh"

namespace meq {
namespace norm {
namespace {

// The weights' place: with two sums over rows per element, 32 elements of a thread leave no registers for them (as
// compiled with them, 92 bytes per thread were spilled and 16384 x 8192 bf16 took 226 us; with them in shared memory 169,
// now 161). Rows that start at different places would need copies at each offset: theirs stay in registers.
template <int kElements, bool kOffset, bool kLayer>
constexpr bool kWeightsShared = kElements > kMostHeld && kLayer && !kOffset;

template <int kElements>
constexpr int threads_of() {
  return kElements > 16 ? 512 : kElements > 8 ? 640 : 1024;
}

// The grid is one cluster, whose blocks add up a share of the columns each, over all blocks in turn; the sums of dy lie
// `second` floats on.
__device__ void add_over_cluster(const BackwardArgs& a, const float* sums, int second) {
  cluster_sync_all();
  for (int v = 0; v < 2; ++v) {
    void* out = v == 0 ? a.dweight : a.dbias;
    if (!out) continue;
    for (int j = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x); j < a.cols; j += static_cast<int>(gridDim.x * blockDim.x)) {
      const uint32_t at = smem_u32(sums + v * second + j);
      float total = 0.f;
      for (uint32_t r = 0; r < gridDim.x; ++r) {
        float x;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(map_to_rank(at, r)) : "memory");
        total += x;
      }
      store_as(out, a.grad_type, j, total);
    }
  }
  cluster_sync_all();  // nobody's sums are read any more
}

template <typename T, int kPieces, bool kOffset, bool kLayer, bool kFew>
__global__ void __launch_bounds__(threads_of<Elem<T>::N * kPieces>(), 1)
    row_backward_kernel(const __grid_constant__ BackwardArgs a, const RowShape s) {
  using P = Place<T, kPieces, kOffset>;
  constexpr int H = P::H, W = P::W;
  constexpr bool kShared = kWeightsShared<2 * H, kOffset, kLayer>;
  pdl_allow_dependents();
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ Exchange ex;
  P p(s);
  const int matrices = a.dh ? 3 : 2, set = kPieces > 1 ? 1 : 32 / s.lanes;  // rows that the group takes at once
  uint8_t* mine = ring + (static_cast<int>(threadIdx.x >> 5) * set + p.sub) * (s.depth * matrices * s.slot_bytes);
  const uint32_t mine32 = smem_u32(mine);
  const uint32_t rows = static_cast<uint32_t>(a.rows), sets = (rows + set - 1) / set, step = gridDim.x * s.groups;
  const uint32_t first = p.group * gridDim.x + blockIdx.x;
  p.set(a.dy, first * set + p.sub, a.ld_dy, a.cols);
  uint32_t next = first;  // set whose copies start next
  int put = 0;
  auto copy_next = [&]() {
    const uint32_t row = next * set + p.sub;
    if (next < sets && row < rows) {
      const uint32_t at = mine32 + static_cast<uint32_t>(put * matrices * s.slot_bytes);
      p.copy(at, a.dy, row, a.ld_dy, a.rows, a.cols);
      p.copy(at + s.slot_bytes, a.h, row, a.ld_h, a.rows, a.cols);
      if (a.dh) p.copy(at + 2 * s.slot_bytes, a.dh, row, a.ld_dh, a.rows, a.cols);
    }
    copies_commit();
    next += step;
    if (++put == s.depth) put = 0;
  };
  auto statistics = [&](uint32_t set_at) -> float2 {  // mu and rstd
    const uint32_t row = set_at * set + p.sub;
    return set_at < sets && row < rows ? make_float2(a.mean ? a.mean[row] : 0.f, a.rstd[row]) : make_float2(0.f, 0.f);
  };
  if (s.warps > 1) clear(ex);
  for (int i = 0; i < s.depth * matrices; ++i) p.clear_slot(mine + i * s.slot_bytes);
  pdl_wait_predecessor();
  for (int i = 0; i < s.depth - 1; ++i) copy_next();
  float2 stat = statistics(first);
  float2 w[kShared ? 1 : H], dw[H], db[kLayer ? H : 1];
  // the thread's columns of the weights, where they are shared
  float4* w_at = reinterpret_cast<float4*>(ring + ring_bytes(s, matrices)) + p.warp_in * (kPieces * 32 * W / 2) + p.lane;
  if constexpr (kShared) {
    if (p.group == 0) {
      float2 v[H];
      p.vector(a.weight, a.weight_type, 1.f, v);
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int e = k * W; e < (k + 1) * W; e += 2) w_at[e / 2 * 32] = make_float4(v[e].x, v[e].y, v[e + 1].x, v[e + 1].y);
    }
    __syncthreads();
  } else {
    p.vector(a.weight, a.weight_type, 1.f, w);
  }
  auto weights = [&](int k, float2 (&v)[W]) {
#pragma unroll
    for (int e = 0; e < W; e += 2) {
      if constexpr (kShared) {
        const float4 q = w_at[(k * W + e) / 2 * 32];
        v[e] = make_float2(q.x, q.y), v[e + 1] = make_float2(q.z, q.w);
      } else {
        v[e] = w[k * W + e], v[e + 1] = w[k * W + e + 1];
      }
    }
  };
#pragma unroll
  for (int k = 0; k < H; ++k) dw[k] = make_float2(0.f, 0.f);
#pragma unroll
  for (int k = 0; k < (kLayer ? H : 1); ++k) db[k] = make_float2(0.f, 0.f);
  const float per = 1.f / static_cast<float>(a.cols);
  int take = 0, turn = 0;
  for (uint32_t i = first; i < sets; i += step) {
    const uint32_t row = i * set + p.sub;
    const bool in = row < rows;
    const float2 now = stat;
    stat = statistics(i + step);
    copies_wait(s.depth);
    copy_next();
    const uint8_t* at = mine + take * matrices * s.slot_bytes;
    if (++take == s.depth) take = 0;
    const float2 mu = make_float2(-now.x, -now.x), rstd = make_float2(now.y, now.y);
    float2 c1 = make_float2(0.f, 0.f), c2 = c1;
    const uint8_t *dy = at, *h = at + s.slot_bytes, *dh = at + 2 * s.slot_bytes;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      float2 x[W], d[W], v[W];
      p.read(h, k, in, x);
      p.read(dy, k, in, d);
      weights(k, v);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int j = k * W + e;
        if (kLayer) x[e] = add2(x[e], mu);
        x[e] = mul2(x[e], rstd);
        dw[j] = fma2(d[e], x[e], dw[j]);
        if (kLayer) db[j] = add2(db[j], d[e]);
        d[e] = mul2(d[e], v[e]);
        c1 = fma2(d[e], x[e], c1);
        if (kLayer) c2 = add2(c2, d[e]);
      }
    }
    float c[kLayer ? 2 : 1] = {c1.x + c1.y};
    if (kLayer) c[kLayer ? 1 : 0] = c2.x + c2.y;
    row_sum<(kLayer ? 2 : 1), (kPieces > 1)>(c, s, p, ex, turn);
    if (!in) continue;
    T* dx = p.at(a.dx, row, a.ld_dx);
    // dx = rstd (a - mean(a) - xhat mean(a xhat)), rstd last: with a tiny eps its square overflows, and so does its product
    // with a mean that xhat would have made small.
    const float s1 = -(c[0] * per), s2 = kLayer && a.mean ? -(c[kLayer ? 1 : 0] * per) : 0.f;
    const float2 m1 = make_float2(s1, s1), m2 = make_float2(s2, s2);
    // dy and h once more from shared memory: kept in registers they would leave no room for the sums.
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      float2 x[W], d[W], v[W];
      p.read(h, k, in, x);
      p.read(dy, k, in, d);
      weights(k, v);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        if (kLayer) x[e] = add2(x[e], mu);
        d[e] = kLayer ? fma2(d[e], v[e], m2) : mul2(d[e], v[e]);
        d[e] = mul2(fma2(mul2(x[e], rstd), m1, d[e]), rstd);
      }
      if (a.dh) {
        p.read(dh, k, in, x);
#pragma unroll
        for (int e = 0; e < W; ++e) d[e] = add2(d[e], x[e]);
      }
      p.write(dx, k, d);
    }
  }
  if (!kFew && !a.parts) return;
  // The block's groups added up, in shared memory: the ring holds 8 bytes for each of their columns.
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  const int copies = s.groups * set, mine_at = p.group * set + p.sub;
  const int wide = s.warps * s.lanes * kPieces * P::N;  // columns with those that do not exist
  float* sums = reinterpret_cast<float*>(ring);
  if (!kOffset) {
#pragma unroll
    for (int k = 0; k < H; k += 2) {
      const int j = p.begin + p.col(k / W) + 2 * (k % W);
      *reinterpret_cast<float4*>(sums + mine_at * wide + j) = make_float4(dw[k].x, dw[k].y, dw[k + 1].x, dw[k + 1].y);
      if (kLayer) *reinterpret_cast<float4*>(sums + (copies + mine_at) * wide + j) = make_float4(db[k].x, db[k].y, db[k + 1].x, db[k + 1].y);
    }
  } else {  // groups whose rows start at different places hold their columns in different pieces
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) {
      const int k = i / P::N, e = i % P::N, j = p.begin + p.col(k) + e;
      if (!p.exists(k, e)) continue;
      sums[mine_at * wide + j] = i % 2 ? dw[i / 2].y : dw[i / 2].x;
      if (kLayer) sums[(copies + mine_at) * wide + j] = i % 2 ? db[i / 2].y : db[i / 2].x;
    }
  }
  __syncthreads();
  const int cols = static_cast<int>(a.cols);
#pragma unroll
  for (int v = 0; v < (kLayer ? 2 : 1); ++v) {
    float* to = kFew ? sums + v * copies * wide : a.parts + (static_cast<int64_t>(v) * gridDim.x + blockIdx.x) * cols;
    for (int j = static_cast<int>(threadIdx.x); j < cols; j += static_cast<int>(blockDim.x)) {
      const float* from = sums + v * copies * wide + j;
      float total = from[0];
#pragma unroll 4
      for (int g = 1; g < copies; ++g) total += from[g * wide];
      to[j] = total;  // few: over the first group's, which this thread alone has read
    }
  }
  if constexpr (kFew) add_over_cluster(a, sums, copies * wide);
}

template <typename T, int kPieces, bool kOffset, bool kLayer, bool kFew>
cudaError_t launch(const BackwardArgs& a, const RowShape& s, int64_t grid, cudaStream_t st) {
  constexpr int kElements = Elem<T>::N * kPieces;
  const int weights = kWeightsShared<kElements, kOffset, kLayer> ? s.warps * s.lanes * kElements * 4 : 0;
  auto* kernel = row_backward_kernel<T, kPieces, kOffset, kLayer, kFew>;
  const cudaError_t e = allow_shared(kernel, kRingBudget);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(32 * s.warps * s.groups), ring_bytes(s, a.dh ? 3 : 2) + weights, st,
                    kFew ? static_cast<int>(grid) : 1, a, s);
}

template <typename T, bool kOffset, bool kLayer, bool kFew>
bool launch_of(const BackwardArgs& a, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  RowShape s;
  int pieces = 0;
  if (!row_shape(a.cols, Elem<T>::N, kOffset, a.dh ? 3 : 2, kLayer, &s, &pieces)) return false;
  const int set = 32 / s.lanes;
  const int64_t sets = (a.rows + set - 1) / set;
  if (kFew) {
    *parts = 1;
    while (*parts < kMostCluster && (*parts < sets || kOffset)) *parts *= 2;
  } else {
    *parts = blocks_for(sets, sms, kOffset);
  }
  *e = pieces == 1   ? launch<T, 1, kOffset, kLayer, kFew>(a, s, *parts, st)
       : pieces == 2 ? launch<T, 2, kOffset, kLayer, kFew>(a, s, *parts, st)
       : pieces == 3 ? launch<T, 3, kOffset, kLayer, kFew>(a, s, *parts, st)
                     : launch<T, 4, kOffset, kLayer, kFew>(a, s, *parts, st);
  return true;
}
template <bool kFew, typename T>
bool launch_of(const BackwardArgs& a, bool layer, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  Starts<T> starts;
  starts.add(a.dy, a.ld_dy, a.rows), starts.add(a.h, a.ld_h, a.rows), starts.add(a.dh, a.ld_dh, a.rows), starts.add(a.dx, a.ld_dx, a.rows);
  if (!starts.alike) return false;
  if (starts.offset || a.cols % Elem<T>::N)
    return layer ? launch_of<T, true, true, kFew>(a, sms, parts, st, e) : launch_of<T, true, false, kFew>(a, sms, parts, st, e);
  return layer ? launch_of<T, false, true, kFew>(a, sms, parts, st, e) : launch_of<T, false, false, kFew>(a, sms, parts, st, e);
}

template <bool kFew>
bool launch_any(const BackwardArgs& a, int type, bool layer, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  if (type == MEQ_F32) return launch_of<kFew, float>(a, layer, sms, parts, st, e);
  if (type == MEQ_BF16) return launch_of<kFew, __nv_bfloat16>(a, layer, sms, parts, st, e);
  return launch_of<kFew, __half>(a, layer, sms, parts, st, e);
}

}  // namespace
}  // namespace norm
}  // namespace meq

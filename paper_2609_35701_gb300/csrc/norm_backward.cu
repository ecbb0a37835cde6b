// The backward pass of the norms: rows that the registers of a group of warps
// hold. One persistent block per SM; dy and h are read once, dx written once, and
// the sums over rows of dy xhat and dy stay in registers until the block's last
// row; then the block's groups are added up and leave one partial sum per column.
#include "norm_rows.cuh"

namespace meq {
namespace norm {
namespace {

// kBias: dy is summed over rows too.
template <int kElements>
constexpr int threads_of() {
  return kElements > 16 ? 512 : kElements > 8 ? 640 : 1024;
}

template <typename T, int kPieces, bool kOffset, bool kBias>
__global__ void __launch_bounds__(threads_of<Elem<T>::N * kPieces>(), 1) row_backward_kernel(const __grid_constant__ BackwardArgs a, const RowShape s) {
  using P = Place<T, kPieces, kOffset>;
  constexpr int H = P::H, W = P::W;
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
  pdl_wait_predecessor();
  for (int i = 0; i < s.depth - 1; ++i) copy_next();
  float2 stat = statistics(first);
  float2 w[H], dw[H], db[kBias ? H : 1];
  p.vector(a.weight, a.weight_type, 1.f, w);
#pragma unroll
  for (int k = 0; k < H; ++k) dw[k] = make_float2(0.f, 0.f);
#pragma unroll
  for (int k = 0; k < (kBias ? H : 1); ++k) db[k] = make_float2(0.f, 0.f);
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
      float2 x[W], d[W];
      p.read(h, k, in, x);
      p.read(dy, k, in, d);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int j = k * W + e;
        x[e] = mul2(add2(x[e], mu), rstd);
        dw[j] = fma2(d[e], x[e], dw[j]);
        if (kBias) db[j] = add2(db[j], d[e]);
        d[e] = mul2(d[e], w[j]);
        c1 = fma2(d[e], x[e], c1);
        c2 = add2(c2, d[e]);
      }
    }
    float c[2] = {c1.x + c1.y, c2.x + c2.y};
    row_sum<2, (kPieces > 1)>(c, s, p, ex, turn);
    const float2 m1 = make_float2(-c[0] * per, -c[0] * per), m2 = a.mean ? make_float2(-c[1] * per, -c[1] * per) : make_float2(0.f, 0.f);
    // dy and h once more from shared memory: kept in registers they would leave no room for the sums.
    if (!in) continue;
    T* dx = p.at(a.dx, row, a.ld_dx);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      float2 x[W], d[W];
      p.read(h, k, in, x);
      p.read(dy, k, in, d);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        x[e] = mul2(add2(x[e], mu), rstd);
        d[e] = mul2(fma2(x[e], m1, fma2(d[e], w[k * W + e], m2)), rstd);
      }
      if (a.dh) {
        p.read(dh, k, in, x);
#pragma unroll
        for (int e = 0; e < W; ++e) d[e] = add2(d[e], x[e]);
      }
      p.write(dx, k, d);
    }
  }
  if (!a.parts) return;
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
      if (kBias) *reinterpret_cast<float4*>(sums + (copies + mine_at) * wide + j) = make_float4(db[k].x, db[k].y, db[k + 1].x, db[k + 1].y);
    }
  } else {  // groups whose rows start at different places hold their columns in different pieces
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) {
      const int k = i / P::N, e = i % P::N, j = p.begin + p.col(k) + e;
      if (!p.exists(k, e)) continue;
      sums[mine_at * wide + j] = i % 2 ? dw[i / 2].y : dw[i / 2].x;
      if (kBias) sums[(copies + mine_at) * wide + j] = i % 2 ? db[i / 2].y : db[i / 2].x;
    }
  }
  __syncthreads();
  const int cols = static_cast<int>(a.cols);
#pragma unroll
  for (int v = 0; v < (kBias ? 2 : 1); ++v) {
    float* to = a.parts + (static_cast<int64_t>(v) * gridDim.x + blockIdx.x) * cols;
    for (int j = static_cast<int>(threadIdx.x); j < cols; j += static_cast<int>(blockDim.x)) {
      const float* from = sums + v * copies * wide + j;
      float total = from[0];
#pragma unroll 4
      for (int g = 1; g < copies; ++g) total += from[g * wide];
      to[j] = total;
    }
  }
}

template <typename T, int kPieces, bool kOffset, bool kBias>
cudaError_t launch(const BackwardArgs& a, const RowShape& s, int64_t grid, cudaStream_t st) {
  auto* kernel = row_backward_kernel<T, kPieces, kOffset, kBias>;
  const cudaError_t e = allow_ring(kernel);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(32 * s.warps * s.groups), ring_bytes(s, a.dh ? 3 : 2), st, 1, a, s);
}

template <typename T, bool kOffset, bool kBias>
bool launch_of(const BackwardArgs& a, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  RowShape s;
  int pieces = 0;
  if (!row_shape(a.cols, Elem<T>::N, kOffset, a.dh ? 3 : 2, &s, &pieces)) return false;
  const int set = 32 / s.lanes;
  const int64_t sets = (a.rows + set - 1) / set;
  *parts = blocks_for(sets, sms, kOffset);
  *e = pieces == 1   ? launch<T, 1, kOffset, kBias>(a, s, *parts, st)
       : pieces == 2 ? launch<T, 2, kOffset, kBias>(a, s, *parts, st)
       : pieces == 3 ? launch<T, 3, kOffset, kBias>(a, s, *parts, st)
                     : launch<T, 4, kOffset, kBias>(a, s, *parts, st);
  return true;
}
template <typename T>
bool launch_of(const BackwardArgs& a, bool bias, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  Starts<T> starts;
  starts.add(a.dy, a.ld_dy, a.rows), starts.add(a.h, a.ld_h, a.rows), starts.add(a.dh, a.ld_dh, a.rows), starts.add(a.dx, a.ld_dx, a.rows);
  if (!starts.alike) return false;
  if (starts.offset || a.cols % Elem<T>::N)
    return bias ? launch_of<T, true, true>(a, sms, parts, st, e) : launch_of<T, true, false>(a, sms, parts, st, e);
  return bias ? launch_of<T, false, true>(a, sms, parts, st, e) : launch_of<T, false, false>(a, sms, parts, st, e);
}

}  // namespace

bool launch_row_backward(const BackwardArgs& a, int type, bool bias, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  if (type == MEQ_F32) return launch_of<float>(a, bias, sms, parts, st, e);
  if (type == MEQ_BF16) return launch_of<__nv_bfloat16>(a, bias, sms, parts, st, e);
  return launch_of<__half>(a, bias, sms, parts, st, e);
}

}  // namespace norm
}  // namespace meq

// Layer norm and RMS norm, forward: rows that the registers of a group of warps
// hold. One persistent block per SM; each row is read once, written once.
//
// Bound by HBM where rows are long and many, us (at the copy rate): RMS norm
// 32768 x 4096 bf16 with a residual 172 (161), layer norm 8192 x 2048 fp32 22.7
// (20.1), 16384 x 2048 bf16 24 (20). Rows that start elsewhere in their 16 bytes
// by latency: 24 elements, weights and biases in a thread's registers leave an SM
// 15 or 16 warps, which issue in half of its slots (0.51) and else wait, each for
// its own last result or for shared memory: 16384 x 2047 40 (20), 6001 x 1025 with
// a residual 17 (7.4). A warp and row take some 300 instructions, and 45 a piece.
#include "norm_rows.cuh"

namespace meq {
namespace norm {
namespace {

template <typename T, int kPieces>
constexpr int threads_of() {
  return Elem<T>::N * kPieces > 16 ? 512 : Elem<T>::N * kPieces > 8 ? 640 : 1024;
}

template <typename T, int kPieces, bool kOffset>
__global__ void __launch_bounds__(threads_of<T, kPieces>(), 1) row_forward_kernel(const __grid_constant__ ForwardArgs a, const RowShape s) {
  using P = Place<T, kPieces, kOffset>;
  constexpr int H = P::H, W = P::W;
  pdl_allow_dependents();
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ Exchange ex;
  P p(s);
  const int matrices = a.residual ? 2 : 1, set = kPieces > 1 ? 1 : 32 / s.lanes;  // rows that the group takes at once
  uint8_t* mine = ring + (static_cast<int>(threadIdx.x >> 5) * set + p.sub) * (s.depth * matrices * s.slot_bytes);
  const uint32_t mine32 = smem_u32(mine);
  const uint32_t rows = static_cast<uint32_t>(a.rows), sets = (rows + set - 1) / set, step = gridDim.x * s.groups;
  const uint32_t first = p.group * gridDim.x + blockIdx.x;
  p.set(a.x, first * set + p.sub, a.ld_x, a.cols);
  uint32_t next = first;  // set whose copies start next
  int put = 0;
  auto copy_next = [&]() {
    const uint32_t row = next * set + p.sub;
    if (next < sets && row < rows) {
      const uint32_t at = mine32 + static_cast<uint32_t>(put * matrices * s.slot_bytes);
      p.copy(at, a.x, row, a.ld_x, a.rows, a.cols);
      if (a.residual) p.copy(at + s.slot_bytes, a.residual, row, a.ld_residual, a.rows, a.cols);
    }
    copies_commit();
    next += step;
    if (++put == s.depth) put = 0;
  };
  if (s.warps > 1) clear(ex);
  for (int i = 0; i < s.depth * matrices; ++i) p.clear_slot(mine + i * s.slot_bytes);
  pdl_wait_predecessor();
  for (int i = 0; i < s.depth - 1; ++i) copy_next();
  float2 w[H], b[H];
  p.vector(a.weight, a.weight_type, 1.f, w);
  p.vector(a.bias, a.weight_type, 0.f, b);
  const float per = 1.f / static_cast<float>(a.cols);
  int take = 0, turn = 0;
  for (uint32_t i = first; i < sets; i += step) {
    const uint32_t row = i * set + p.sub;
    const bool in = row < rows;
    copies_wait(s.depth);
    copy_next();
    const uint8_t* at = mine + take * matrices * s.slot_bytes;
    if (++take == s.depth) take = 0;
    float2 v[H];
    T* h = p.at(a.h, row, a.ld_h);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      float2 x[W];
      p.read(at, k, in, x);
      if (a.residual) {
        float2 r[W];
        p.read(at + s.slot_bytes, k, in, r);
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = round_pair<T>(add2(x[e], r[e]));
        if (in) p.write(h, k, x);
      }
#pragma unroll
      for (int e = 0; e < W; ++e) v[k * W + e] = x[e];
    }
    float mu = 0.f;
    if (a.mean) {
      float2 sum = v[0];
#pragma unroll
      for (int k = 1; k < H; ++k) sum = add2(sum, v[k]);
      float total[1] = {sum.x + sum.y};
      row_sum<1, (kPieces > 1)>(total, s, p, ex, turn);
      mu = total[0] * per;
#pragma unroll
      for (int k = 0; k < H; ++k) v[k] = add2(v[k], make_float2(-mu, -mu));
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (!p.has(k) || p.part(k)) p.clip(k, v + k * W);
    }
    float2 sq = mul2(v[0], v[0]);
#pragma unroll
    for (int k = 1; k < H; ++k) sq = fma2(v[k], v[k], sq);
    float total[1] = {sq.x + sq.y};
    row_sum<1, (kPieces > 1)>(total, s, p, ex, turn);
    const float rstd = inverse_root(total[0] * per, a.eps);
    if (!in) continue;
    T* y_row = p.at(a.y, row, a.ld_y);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      float2 y[W];
#pragma unroll
      for (int e = 0; e < W; ++e) y[e] = fma2(mul2(v[k * W + e], make_float2(rstd, rstd)), w[k * W + e], b[k * W + e]);
      p.write(y_row, k, y);
    }
    if (p.warp_in == 0 && p.lane == 0) {
      if (a.mean) a.mean[row] = mu;
      a.rstd[row] = rstd;
    }
  }
}

template <typename T, int kPieces, bool kOffset>
cudaError_t launch(const ForwardArgs& a, const RowShape& s, int sms, cudaStream_t st) {
  const int set = 32 / s.lanes;
  const int64_t sets = (a.rows + set - 1) / set;
  auto* kernel = row_forward_kernel<T, kPieces, kOffset>;
  const cudaError_t e = allow_shared(kernel, kRingBudget);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(blocks_for(sets, sms, kOffset)), dim3(32 * s.warps * s.groups), ring_bytes(s, a.residual ? 2 : 1),
                    st, 1, a, s);
}

template <typename T, bool kOffset>
bool launch_of(const ForwardArgs& a, int sms, cudaStream_t st, cudaError_t* e) {
  RowShape s;
  int pieces = 0;
  if (!row_shape(a.cols, Elem<T>::N, kOffset, a.residual ? 2 : 1, false, &s, &pieces)) return false;
  *e = pieces == 1   ? launch<T, 1, kOffset>(a, s, sms, st)
       : pieces == 2 ? launch<T, 2, kOffset>(a, s, sms, st)
       : pieces == 3 ? launch<T, 3, kOffset>(a, s, sms, st)
                     : launch<T, 4, kOffset>(a, s, sms, st);
  return true;
}
template <typename T>
bool launch_of(const ForwardArgs& a, int sms, cudaStream_t st, cudaError_t* e) {
  Starts<T> starts;
  starts.add(a.x, a.ld_x, a.rows), starts.add(a.y, a.ld_y, a.rows), starts.add(a.residual, a.ld_residual, a.rows), starts.add(a.h, a.ld_h, a.rows);
  if (!starts.alike) return false;
  return starts.offset || a.cols % Elem<T>::N ? launch_of<T, true>(a, sms, st, e) : launch_of<T, false>(a, sms, st, e);
}

}  // namespace

bool launch_row_forward(const ForwardArgs& a, int type, int sms, cudaStream_t st, cudaError_t* e) {
  if (type == MEQ_F32) return launch_of<float>(a, sms, st, e);
  if (type == MEQ_BF16) return launch_of<__nv_bfloat16>(a, sms, st, e);
  return launch_of<__half>(a, sms, st, e);
}

}  // namespace norm
}  // namespace meq

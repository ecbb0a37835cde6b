// Layer norm and RMS norm, forward: rows that the registers of a group of warps
// hold. One persistent block per SM; each row is read once, written once.
#include "norm_rows.cuh"

namespace meq {
namespace norm {
namespace {

template <typename T, int kStep, int kPieces>
constexpr int threads_of() {
  return kStep * kPieces > 16 ? 512 : kStep * kPieces > 8 ? 640 : 1024;
}

template <typename T, int kStep, int kPieces>
__global__ void __launch_bounds__(threads_of<T, kStep, kPieces>(), 1) row_forward_kernel(const __grid_constant__ ForwardArgs a, const RowShape s) {
  using P = Place<T, kStep, kPieces>;
  constexpr int H = P::H;
  pdl_allow_dependents();
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ Exchange ex;
  const P p(s, a.cols);
  const int matrices = a.residual ? 2 : 1, set = 32 / s.lanes;  // rows that the group takes at once
  const int slots = s.depth * matrices * s.slot_bytes;
  uint8_t* mine = ring + static_cast<int64_t>(p.group * set + p.sub) * slots;
  const uint32_t mine32 = smem_u32(mine);
  const int64_t sets = (a.rows + set - 1) / set, step = static_cast<int64_t>(gridDim.x) * s.groups;
  int64_t next = static_cast<int64_t>(p.group) * gridDim.x + blockIdx.x;  // set whose copies start next
  int put = 0;
  auto copy_next = [&]() {
    const int64_t row = next * set + p.sub;
    if (next < sets && row < a.rows) {
      const uint32_t at = mine32 + static_cast<uint32_t>(put * matrices * s.slot_bytes);
      p.copy(at, a.x, row, a.ld_x, a.rows);
      if (a.residual) p.copy(at + s.slot_bytes, a.residual, row, a.ld_residual, a.rows);
    }
    copies_commit();
    next += step;
    if (++put == s.depth) put = 0;
  };
  pdl_wait_predecessor();
  for (int i = 0; i < s.depth - 1; ++i) copy_next();
  float2 w[H], b[H];
  p.vector(a.weight, a.weight_type, a.weight ? 0.f : 1.f, w);
  p.vector(a.bias, a.weight_type, 0.f, b);
  const float per = 1.f / static_cast<float>(a.cols);
  int take = 0, turn = 0;
  for (int64_t i = static_cast<int64_t>(p.group) * gridDim.x + blockIdx.x; i < sets; i += step) {
    const int64_t row = i * set + p.sub;
    const bool in = row < a.rows;
    copies_wait(s.depth);
    if (kStep == 1) group_barrier(s, p.group);  // the others' copies too, and the slot before is free
    copy_next();
    const uint8_t* at = mine + take * matrices * s.slot_bytes;
    if (++take == s.depth) take = 0;
    float2 v[H];
    const uint8_t* x = p.row_at(at, a.x, row, a.ld_x);
    const uint8_t* r = p.row_at(at + s.slot_bytes, a.residual, row, a.ld_residual);
#pragma unroll
    for (int u = 0; u < P::U; ++u) {
      float2 y[P::W];
      p.read(x, u, in, y);
      if (a.residual) {
        float2 z[P::W];
        p.read(r, u, in, z);
#pragma unroll
        for (int k = 0; k < P::W; ++k) y[k] = round_pair<T>(add2(y[k], z[k]));
        if (in) p.write(static_cast<T*>(a.h) + row * a.ld_h, u, y);
      }
#pragma unroll
      for (int k = 0; k < P::W; ++k) v[u * P::W + k] = y[k];
    }
    float mu = 0.f;
    if (a.mean) {
      float2 sum = v[0];
#pragma unroll
      for (int k = 1; k < H; ++k) sum = add2(sum, v[k]);
      mu = row_sum(make_float2(sum.x + sum.y, 0.f), s, p.group, p.warp_in, ex, turn).x * per;
#pragma unroll
      for (int k = 0; k < H; ++k) v[k] = add2(v[k], make_float2(-mu, -mu));
      p.clip(v);
    }
    float2 sq = mul2(v[0], v[0]);
#pragma unroll
    for (int k = 1; k < H; ++k) sq = fma2(v[k], v[k], sq);
    const float var = row_sum(make_float2(sq.x + sq.y, 0.f), s, p.group, p.warp_in, ex, turn).x * per;
    const float rstd = inverse_root(var, a.eps);
    if (!in) continue;
#pragma unroll
    for (int k = 0; k < H; ++k) v[k] = fma2(mul2(v[k], make_float2(rstd, rstd)), w[k], b[k]);
#pragma unroll
    for (int u = 0; u < P::U; ++u) p.write(static_cast<T*>(a.y) + row * a.ld_y, u, v + u * P::W);
    if (p.t == 0) {
      if (a.mean) a.mean[row] = mu;
      a.rstd[row] = rstd;
    }
  }
}

template <typename T, int kStep, int kPieces>
cudaError_t launch(const ForwardArgs& a, const RowShape& s, int sms, cudaStream_t st) {
  const int set = 32 / s.lanes, bytes = ring_bytes(s, a.residual ? 2 : 1);
  const int64_t sets = (a.rows + set - 1) / set;
  auto* kernel = row_forward_kernel<T, kStep, kPieces>;
  const cudaError_t e = allow_ring(kernel);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(sets < sms ? sets : sms)), dim3(32 * s.warps * s.groups), bytes, st, 1, a, s);
}

template <typename T>
bool launch_of(const ForwardArgs& a, int sms, cudaStream_t st, cudaError_t* e) {
  constexpr int kN = Elem<T>::N;
  const int matrices = a.residual ? 2 : 1;
  const bool whole = a.cols % kN == 0 && starts_at_16<T>(a.x, a.ld_x) && starts_at_16<T>(a.y, a.ld_y) && starts_at_16<T>(a.residual, a.ld_residual) &&
                     starts_at_16<T>(a.h, a.ld_h);
  RowShape s;
  int pieces = 0;
  if (whole) {
    if (!row_shape(a.cols, kN, sizeof(T), matrices, false, kWholePieces, 4, &s, &pieces)) return false;
    *e = pieces == 1   ? launch<T, kN, 1>(a, s, sms, st)
         : pieces == 2 ? launch<T, kN, 2>(a, s, sms, st)
         : pieces == 3 ? launch<T, kN, 3>(a, s, sms, st)
                       : launch<T, kN, 4>(a, s, sms, st);
  } else {
    if (!row_shape(a.cols, 1, sizeof(T), matrices, false, kSingles, 4, &s, &pieces)) return false;
    *e = pieces == 2    ? launch<T, 1, 2>(a, s, sms, st)
         : pieces == 8  ? launch<T, 1, 8>(a, s, sms, st)
         : pieces == 16 ? launch<T, 1, 16>(a, s, sms, st)
                        : launch<T, 1, 32>(a, s, sms, st);
  }
  return true;
}

}  // namespace

bool launch_row_forward(const ForwardArgs& a, int type, int sms, cudaStream_t st, cudaError_t* e) {
  if (type == MEQ_F32) return launch_of<float>(a, sms, st, e);
  if (type == MEQ_BF16) return launch_of<__nv_bfloat16>(a, sms, st, e);
  return launch_of<__half>(a, sms, st, e);
}

}  // namespace norm
}  // namespace meq

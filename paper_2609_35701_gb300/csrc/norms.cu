// Layer norm and RMS norm, with the addition to the residual stream, and their
// backward pass.
//
// Forward, per row:  h = x + residual (rounded to its type),
//   mu = mean(h) (RMS: 0), rstd = 1 / sqrt(mean((h - mu)^2) + eps),
//   y = (h - mu) rstd w + b.
// Backward, with xhat = (h - mu) rstd and a = dy w:
//   dx = rstd (a - mean(a) - xhat mean(a xhat)) (+ dh; RMS: no mean(a)),
//   dw = sum over rows of dy xhat,  db = sum over rows of dy.
//
// The variance is that of differences from the mean, not a difference of
// squares. Sums are fp32, in fixed orders.
#include <string>

#include "meq_call.cuh"
#include "norm_rows.cuh"

namespace meq {
namespace norm {
namespace {

constexpr int kWideThreads = 512;
constexpr int kWideWarps = kWideThreads / 32;
constexpr int kTileThreads = 128;     // of a block of the wide rows' gradient
constexpr int64_t kMostParts = 192;   // partial sums of a column, at most
constexpr int64_t kPartFloats = kMostParts * 16384;
constexpr int kFoldSlices = 32;
// Up to so many elements one cluster takes the rows and adds up the sums over them itself: a launch less, which takes the
// host as long as the rows take the GPU (24 x 768 fp32: 3.4 us on the GPU for 4.1, 17 on the host for 21). 64 x 1024
// bf16 takes 6.6 us for 7.2, but 1000 x 65 11.3 for 8.4 on the GPU; with 256 x 1024 the cluster would take 10.6 for 7.7.
constexpr int64_t kFewElements = 65536;

// The sum of a block's values, for every thread; sh is free again after the next barrier.
__device__ __forceinline__ float block_sum(float x, float* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kWideWarps; ++i) s += sh[i];
  return s;
}

// kStep elements from column j on: a 16-byte piece, or one.
template <typename T, int kStep>
__device__ __forceinline__ void load(const T* p, int64_t j, float (&x)[kStep]) {
  if constexpr (kStep == 1) {
    x[0] = Elem<T>::get(p + j);
  } else {
    float2 y[kStep / 2];
    Elem<T>::unpack(*reinterpret_cast<const uint4*>(p + j), y);
#pragma unroll
    for (int e = 0; e < kStep / 2; ++e) x[2 * e] = y[e].x, x[2 * e + 1] = y[e].y;
  }
}
template <typename T, int kStep>
__device__ __forceinline__ void store(T* p, int64_t j, const float (&x)[kStep]) {
  if constexpr (kStep == 1) {
    p[j] = Elem<T>::make(x[0]);
  } else {
    float2 y[kStep / 2];
#pragma unroll
    for (int e = 0; e < kStep / 2; ++e) y[e] = make_float2(x[2 * e], x[2 * e + 1]);
    *reinterpret_cast<uint4*>(p + j) = Elem<T>::pack(y);
  }
}

// Rows that no group of warps holds: a block per row, which it reads again for each step (from L2, but for very long
// ones). 2000 x 16384 fp32 84 us (39 at the copy rate), its backward pass, which reads dy and h twice, 126 (59). Matrices
// whose rows lie in their 16 bytes differently come here too, an element per lane and load: 16384 x 2047 bf16 into rows of
// 2048 125 us (40 into rows of 2047; 20 at the copy rate), backward 231 (67; 30).
template <typename T, int kStep>
__global__ void __launch_bounds__(kWideThreads) wide_forward_kernel(const ForwardArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ float sh[2][kWideWarps];
  const int64_t first = threadIdx.x * kStep, step = kWideThreads * kStep;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    T* y = static_cast<T*>(a.y) + row * a.ld_y;
    float sum = 0.f, v[kStep];
    if (a.residual) {
      const T* r = static_cast<const T*>(a.residual) + row * a.ld_residual;
      T* h = static_cast<T*>(a.h) + row * a.ld_h;
      for (int64_t j = first; j < a.cols; j += step) {
        float z[kStep];
        load(x, j, v);
        load(r, j, z);
#pragma unroll
        for (int e = 0; e < kStep; ++e) {
          const T held = Elem<T>::make(v[e] + z[e]);
          v[e] = Elem<T>::get(&held);
          sum += v[e];
        }
        store(h, j, v);
      }
      x = h;
    } else if (a.mean) {
#pragma unroll 4
      for (int64_t j = first; j < a.cols; j += step) {
        load(x, j, v);
#pragma unroll
        for (int e = 0; e < kStep; ++e) sum += v[e];
      }
    }
    const float n = static_cast<float>(a.cols);
    const float mu = a.mean ? block_sum(sum, sh[0]) / n : 0.f;
    float sq = 0.f;
#pragma unroll 4
    for (int64_t j = first; j < a.cols; j += step) {
      load(x, j, v);
#pragma unroll
      for (int e = 0; e < kStep; ++e) sq = fmaf(v[e] - mu, v[e] - mu, sq);
    }
    const float rstd = inverse_root(block_sum(sq, sh[1]) / n, a.eps);
#pragma unroll 2
    for (int64_t j = first; j < a.cols; j += step) {
      load(x, j, v);
#pragma unroll
      for (int e = 0; e < kStep; ++e) {
        v[e] = (v[e] - mu) * rstd;
        if (a.weight) v[e] *= load_as(a.weight, a.weight_type, j + e);
        if (a.bias) v[e] += load_as(a.bias, a.weight_type, j + e);
      }
      store(y, j, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mu;
      a.rstd[row] = rstd;
    }
    __syncthreads();
  }
}

// mean(a xhat) and mean(a) of a row per block.
template <typename T, int kStep>
__global__ void __launch_bounds__(kWideThreads) wide_sums_kernel(const BackwardArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ float sh[2][kWideWarps];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* h = static_cast<const T*>(a.h) + row * a.ld_h;
    const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
    float c1 = 0.f, c2 = 0.f;
#pragma unroll 2
    for (int64_t j = threadIdx.x * kStep; j < a.cols; j += kWideThreads * kStep) {
      float d[kStep], x[kStep];
      load(dy, j, d);
      load(h, j, x);
#pragma unroll
      for (int e = 0; e < kStep; ++e) {
        if (a.weight) d[e] *= load_as(a.weight, a.weight_type, j + e);
        c1 = fmaf(d[e], (x[e] - mu) * rstd, c1);
        c2 += d[e];
      }
    }
    c1 = block_sum(c1, sh[0]);
    c2 = block_sum(c2, sh[1]);
    if (threadIdx.x == 0) {
      const float n = static_cast<float>(a.cols);
      a.row_sums[2 * row] = c1 / n;
      a.row_sums[2 * row + 1] = a.mean ? c2 / n : 0.f;
    }
    __syncthreads();
  }
}

// A thread per kStep columns, over every gridDim.y-th row: dx, and the columns' partial sums.
template <typename T, int kStep>
__global__ void __launch_bounds__(kTileThreads) wide_backward_kernel(const BackwardArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const int64_t j = (static_cast<int64_t>(blockIdx.x) * kTileThreads + threadIdx.x) * kStep;
  if (j >= a.cols) return;
  float w[kStep], dw[kStep], db[kStep];
#pragma unroll
  for (int e = 0; e < kStep; ++e) w[e] = a.weight ? load_as(a.weight, a.weight_type, j + e) : 1.f, dw[e] = db[e] = 0.f;
#pragma unroll 2
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float mu = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row], c1 = a.row_sums[2 * row], c2 = a.row_sums[2 * row + 1];
    float d[kStep], x[kStep], r[kStep] = {};
    load(static_cast<const T*>(a.dy) + row * a.ld_dy, j, d);
    load(static_cast<const T*>(a.h) + row * a.ld_h, j, x);
    if (a.dh) load(static_cast<const T*>(a.dh) + row * a.ld_dh, j, r);
#pragma unroll
    for (int e = 0; e < kStep; ++e) {
      const float xhat = (x[e] - mu) * rstd;
      dw[e] = fmaf(d[e], xhat, dw[e]);
      db[e] += d[e];
      r[e] += rstd * (fmaf(d[e], w[e], -c2) - xhat * c1);
    }
    store(static_cast<T*>(a.dx) + row * a.ld_dx, j, r);
  }
  if (!a.parts) return;
#pragma unroll
  for (int e = 0; e < kStep; ++e) {
    a.parts[static_cast<int64_t>(blockIdx.y) * a.cols + j + e] = dw[e];
    a.parts[(static_cast<int64_t>(gridDim.y) + blockIdx.y) * a.cols + j + e] = db[e];
  }
}

// dw and db (blockIdx.y) from the partial sums, 32 columns per block. A warp takes
// every 32nd part, at most 6 of them, all on their way at once: 4096 columns of
// 152 parts take 5 us alone, a launch and two trips to memory (in a chain, 19
// parts a thread, 9.5).
__global__ void __launch_bounds__(32 * kFoldSlices) fold_parts_kernel(const float* parts, int64_t n, int64_t cols, void* dw, void* db, int type) {
  pdl_allow_dependents();
  __shared__ float sh[kFoldSlices][33];
  const int lane = static_cast<int>(threadIdx.x & 31), slice = static_cast<int>(threadIdx.x >> 5);
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  void* out = blockIdx.y == 0 ? dw : db;
  const float* p = parts + static_cast<int64_t>(blockIdx.y) * n * cols + j;
  pdl_wait_predecessor();
  if (!out) return;
  constexpr int kEach = static_cast<int>((kMostParts + kFoldSlices - 1) / kFoldSlices);
  float x[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int64_t i = slice + k * kFoldSlices;
    x[k] = i < n && j < cols ? p[i * cols] : 0.f;
  }
  float s = x[0];
#pragma unroll
  for (int k = 1; k < kEach; ++k) s += x[k];
  sh[slice][lane] = s;
  __syncthreads();
  // warp w adds up column w: lane l's slice is l
  s = sh[lane][slice];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + slice;
  if (lane == 0 && c < cols) store_as(out, type, c, s);
}

// ------------------------------------------------------------------- host
int64_t parts_for(int64_t rows, int64_t cols) {
  int64_t n = kPartFloats / cols;
  if (n > kMostParts) n = kMostParts;
  if (n > (rows + 7) / 8 * 8) n = (rows + 7) / 8 * 8;
  return n < 1 ? 1 : n;
}

unsigned row_grid(int64_t rows) { return static_cast<unsigned>(rows < (1 << 30) ? rows : (1 << 30)); }

template <typename T>
cudaError_t launch_wide_forward(const ForwardArgs& a, cudaStream_t st) {
  Starts<T> starts;
  starts.add(a.x, a.ld_x, a.rows), starts.add(a.y, a.ld_y, a.rows), starts.add(a.residual, a.ld_residual, a.rows), starts.add(a.h, a.ld_h, a.rows);
  const bool whole = !starts.offset && a.cols % Elem<T>::N == 0;
  return launch_pdl(whole ? wide_forward_kernel<T, Elem<T>::N> : wide_forward_kernel<T, 1>, dim3(row_grid(a.rows)), dim3(kWideThreads), 0, st, 1, a);
}

template <typename T, int kStep>
cudaError_t launch_wide_backward(const BackwardArgs& a, int64_t parts, cudaStream_t st) {
  const cudaError_t e = launch_pdl(wide_sums_kernel<T, kStep>, dim3(row_grid(a.rows)), dim3(kWideThreads), 0, st, 1, a);
  if (e != cudaSuccess) return e;
  constexpr int64_t cols = kTileThreads * kStep;
  return launch_pdl(wide_backward_kernel<T, kStep>, dim3(static_cast<unsigned>((a.cols + cols - 1) / cols), static_cast<unsigned>(parts)),
                    dim3(kTileThreads), 0, st, 1, a);
}
template <typename T>
cudaError_t launch_wide_backward(const BackwardArgs& a, int64_t* parts, cudaStream_t st) {
  Starts<T> starts;
  starts.add(a.dy, a.ld_dy, a.rows), starts.add(a.h, a.ld_h, a.rows), starts.add(a.dh, a.ld_dh, a.rows), starts.add(a.dx, a.ld_dx, a.rows);
  *parts = parts_for(a.rows, a.cols);
  if (!starts.offset && a.cols % Elem<T>::N == 0) return launch_wide_backward<T, Elem<T>::N>(a, *parts, st);
  return launch_wide_backward<T, 1>(a, *parts, st);
}

// The checks that both calls share; an empty text: fine.
std::string check_shape(int type, int64_t rows, int64_t cols, int weight_type) {
  if (!valid_type(type) || !valid_type(weight_type)) return "the types must be meq_dtypes";
  if (rows < 0 || rows > (int64_t(1) << 27)) return "rows must be in 0..2^27";
  if (cols < 1 || cols > (int64_t(1) << 20)) return "cols must be in 1..2^20";
  return "";
}
std::string check_matrix(const void* p, int64_t ld, int type, int64_t rows, int64_t cols, const char* what, bool needed) {
  if (!p) return needed && rows > 0 ? std::string(what) + " must not be NULL" : "";
  if (!aligned_to(p, elem_bytes(type))) return std::string(what) + " is not aligned to its type";
  if (rows > 1 && ld < cols) return "the row stride of " + std::string(what) + " must be at least cols";
  if (ld < 0 || ld > (int64_t(1) << 40)) return "the row stride of " + std::string(what) + " must be in 0..2^40";
  return "";
}

}  // namespace
}  // namespace norm
}  // namespace meq

using namespace meq;
using namespace meq::norm;

extern "C" {

meq_status meq_layer_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int type, int64_t rows, int64_t cols,
                          const void* weight, const void* bias, int weight_type, float eps, void* y, int64_t ld_y, void* h, int64_t ld_h,
                          float* mean, float* rstd, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_shape(type, rows, cols, weight_type);
    if (why.empty()) why = check_matrix(x, ld_x, type, rows, cols, "x", true);
    if (why.empty()) why = check_matrix(residual, ld_residual, type, rows, cols, "residual", false);
    if (why.empty()) why = check_matrix(y, ld_y, type, rows, cols, "y", true);
    if (why.empty()) why = check_matrix(h, ld_h, type, rows, cols, "h", residual != nullptr);
    if (why.empty() && h && !residual) why = "h is written with a residual only";
    if (why.empty() && h && h == y) why = "y and h must not be the same";
    if (why.empty() && !(eps > 0.f && eps <= FLT_MAX)) why = "eps must be finite and > 0";
    if (why.empty() && rows > 0 && !rstd) why = "rstd must not be NULL";
    if (why.empty() && !(aligned_to(weight, elem_bytes(weight_type)) && aligned_to(bias, elem_bytes(weight_type)) && aligned_to(mean, 4) &&
                         aligned_to(rstd, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_layer_norm: " + why);
    if (rows == 0) return MEQ_OK;
    ForwardArgs a{};
    a.x = x, a.residual = residual, a.weight = weight, a.bias = bias, a.y = y, a.h = h, a.mean = mean, a.rstd = rstd;
    a.rows = rows, a.cols = cols, a.ld_x = ld_x, a.ld_residual = ld_residual, a.ld_y = ld_y, a.ld_h = ld_h;
    a.weight_type = weight_type, a.eps = eps;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_layer_norm", "device attributes");
    if (!launch_row_forward(a, type, sms, st, &e))
      e = type == MEQ_F32    ? launch_wide_forward<float>(a, st)
          : type == MEQ_BF16 ? launch_wide_forward<__nv_bfloat16>(a, st)
                             : launch_wide_forward<__half>(a, st);
    return launch_status(e, "meq_layer_norm", "launch");
  });
}

int64_t meq_layer_norm_work_floats(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1) return 0;
  return 2 * parts_for(rows, cols) * cols + 2 * rows;
}

meq_status meq_layer_norm_grad(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* dh, int64_t ld_dh, int type,
                               int64_t rows, int64_t cols, const void* weight, int weight_type, const float* mean, const float* rstd,
                               void* dx, int64_t ld_dx, void* dweight, void* dbias, int grad_type, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_shape(type, rows, cols, weight_type);
    if (why.empty() && !valid_type(grad_type)) why = "the types must be meq_dtypes";
    if (why.empty()) why = check_matrix(dy, ld_dy, type, rows, cols, "dy", true);
    if (why.empty()) why = check_matrix(h, ld_h, type, rows, cols, "h", true);
    if (why.empty()) why = check_matrix(dh, ld_dh, type, rows, cols, "dh", false);
    if (why.empty()) why = check_matrix(dx, ld_dx, type, rows, cols, "dx", true);
    if (why.empty() && rows > 0 && !rstd) why = "rstd must not be NULL";
    if (why.empty() && (!aligned_to(work, 16) || (!work && rows * cols > kFewElements))) why = "work must not be NULL and be 16-byte aligned";
    if (why.empty() && !(aligned_to(weight, elem_bytes(weight_type)) && aligned_to(dweight, elem_bytes(grad_type)) &&
                         aligned_to(dbias, elem_bytes(grad_type)) && aligned_to(mean, 4) && aligned_to(rstd, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_layer_norm_grad: " + why);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    BackwardArgs a{};
    a.dy = dy, a.h = h, a.dh = dh, a.weight = weight, a.mean = mean, a.rstd = rstd, a.dx = dx;
    a.rows = rows, a.cols = cols, a.ld_dy = ld_dy, a.ld_h = ld_h, a.ld_dh = ld_dh, a.ld_dx = ld_dx;
    a.weight_type = weight_type, a.parts = dweight || dbias ? work : nullptr, a.row_sums = work ? work + 2 * parts_for(rows, cols) * cols : nullptr;
    int64_t parts = 0;
    if (rows > 0) {
      cudaError_t e;
      int sms = device_sms(&e);
      if (e != cudaSuccess) return launch_status(e, "meq_layer_norm_grad", "device attributes");
      if (sms > kMostParts) sms = kMostParts;  // what work has room for
      const bool wanted = dweight || dbias;
      if (wanted && rows * cols <= kFewElements) {
        a.dweight = dweight, a.dbias = dbias, a.grad_type = grad_type;
        if (launch_few_backward(a, type, mean || dbias, st, &e)) return launch_status(e, "meq_layer_norm_grad", "launch");
      }
      const bool in_registers = (work || !wanted) && launch_row_backward(a, type, mean || dbias, sms, &parts, st, &e);
      if (!in_registers && !work)
        return fail(MEQ_ERR_INVALID_ARG, "meq_layer_norm_grad: these rows need work (they are too long, or lie in their 16 bytes differently)");
      if (!in_registers)
        e = type == MEQ_F32    ? launch_wide_backward<float>(a, &parts, st)
            : type == MEQ_BF16 ? launch_wide_backward<__nv_bfloat16>(a, &parts, st)
                               : launch_wide_backward<__half>(a, &parts, st);
      if (e != cudaSuccess) return launch_status(e, "meq_layer_norm_grad", "launch");
    }
    if (!dweight && !dbias) return MEQ_OK;
    const dim3 grid(static_cast<unsigned>((cols + 31) / 32), dbias ? 2u : 1u);
    return launch_status(launch_pdl(fold_parts_kernel, grid, dim3(32 * kFoldSlices), 0, st, 1, static_cast<const float*>(work), parts, cols,
                                    dweight, dbias, grad_type),
                         "meq_layer_norm_grad", "sum launch");
  });
}

}  // extern "C"

// Losses of fine-tuning on token log-probabilities, and the gradient of the
// logits: token log-probabilities, the clipped policy loss with its KL term,
// and the paired preference loss.
//
// For a row of logits z with target t:  lse = log sum_j exp(z_j),
// logp = z_t - lse,  d logp / d z_j = [j = t] - exp(z_j - lse). Every loss here
// is a function of the rows' logp, so the gradient of a row is one coefficient
// c = dL/dlogp times ([j = t] - softmax_j).
//
// HBM bounds all of them: two exponentials per element stand against 4 bytes
// moved (bf16, with the gradient).
//
// Policy loss: c depends on the row alone, so a row is read once, kept on chip
// and its gradient written from there: the floor. Few or short rows are held in
// registers (8 pieces of 16 bytes per thread) by one CTA or a cluster of up to
// 8, reduced (warp, CTA, then the cluster's CTAs through distributed shared
// memory): 4096 x 16000 bf16 48 us (39 at the measured copy rate, 6.79 TB/s).
// Many long ones are streamed through shared memory, in a file of their own.
// Rows that neither holds take three launches (statistics, coefficients,
// gradient): 256 x 600000 bf16 151 us (136 for two reads and a write).
//
// Preference loss: c needs the sums over the two answers of a pair, so the
// logits are read again for the gradient, last rows first: those are the ones
// that the statistics pass left in L2. 9600 x 32000 bf16 309 us (272 for two
// reads and a write at the copy rate).
//
// Rows start at any element: a row is cut at the 16-byte boundaries of its
// address, and only its first and last piece are moved element by element.
// Sums and statistics are fp32 or wider; exponentials are of z - max.
#include <new>
#include <string>

#include "loss_rows.cuh"
#include "meq_mbar.cuh"

using namespace meq;
using namespace meq::loss;

namespace {

constexpr int kPieces = 8;          // 16-byte pieces per thread
constexpr int kChunkPieces = 32 * kPieces;  // of a warp
constexpr int kMaxCluster = 8;
constexpr int kShortThreads = 128;
constexpr int kShortPerSm = 64;     // blocks per SM at most (1000000 x 256 bf16: 16, 64, any number, us: 565, 550, 637)
constexpr int kRowThreads = 512;    // most threads of a CTA before the cluster grows
constexpr int kRowThreadsMax = 1024;
// 16-byte pieces per thread and threads of the gradient pass: 8 KB of a row per
// block. 9600 x 32000 bf16, pieces x threads 4 x 128, 4 x 256, 8 x 256, 2 x 256,
// 4 x 512, us: 212, 213, 215, 213, 219; 2048 x 50001 fp32 147, 148, 151, 149, 155.
constexpr int kGradThreads = 128;
constexpr int kGradPieces = 4;

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}

struct RowShared {
  MaxSum warp[32];
  MaxSum cta[kMaxCluster];
};

// The maximum and sum of the whole row from each warp's, for every thread of
// the cluster, in an order that does not depend on timing.
__device__ __forceinline__ MaxSum row_join(MaxSum w, RowShared& sh, uint32_t rank, uint32_t ctas) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) sh.warp[threadIdx.x >> 5] = w;
  __syncthreads();
  MaxSum t{-INFINITY, 0.f};
  if (lane < warps) t = sh.warp[lane];
  const float m = warp_max(t.m);
  t.s *= exp_diff(t.m, finite_or_zero(m));
  t.m = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t.s += __shfl_xor_sync(0xffffffffu, t.s, o);
  if (ctas == 1) return t;
  // every CTA of the cluster has begun (the wait of the arrive at the kernel's start)
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (threadIdx.x < ctas) {
    const uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(&sh.cta[rank]));
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(remote), "f"(t.m), "f"(t.s) : "memory");
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  MaxSum r = sh.cta[0];
  for (uint32_t i = 1; i < ctas; ++i) r = join(r, sh.cta[i]);
  return r;
}

// max and sum of exponentials over a warp's pieces, for all its lanes
template <typename T, int P>
__device__ __forceinline__ MaxSum warp_stats(const uint4 (&q)[P]) {
  MaxSum w;
  typename Elem<T>::Max top = Elem<T>::none();
#pragma unroll
  for (int j = 0; j < P; ++j) top = Elem<T>::max_of(top, q[j]);
  const float m = warp_max(Elem<T>::value(top));
  w.m = m;
  constexpr int H = Elem<T>::N / 2;
  float2 s = make_float2(0.f, 0.f);
  float own = 1.f, fix = 1.f;  // the maximum's own term as it is in the sum
  if (fabsf(m) <= kFar || m == -INFINITY) {
    const ExpBase b(finite_or_zero(m));
    own = exp_at(m, b.c), fix = b.fix;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float2 x[H];
      Elem<T>::unpack(q[j], x);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const float2 y = fma2(x[e], make_float2(kLog2e, kLog2e), make_float2(-b.c, -b.c));
        const float2 z = fma2(x[e], make_float2(kLog2eLo, kLog2eLo), y);
        s = add2(s, make_float2(exp2_approx(z.x), exp2_approx(z.y)));
      }
    }
  } else {
    // far from zero (+inf gives NaN)
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float2 x[H];
      Elem<T>::unpack(q[j], x);
#pragma unroll
      for (int e = 0; e < H; ++e) s = add2(s, make_float2(exp_diff(x[e].x, m), exp_diff(x[e].y, m)));
    }
  }
  w.s = s.x + s.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) w.s += __shfl_xor_sync(0xffffffffu, w.s, o);
  if (m != -INFINITY) w.s = fmaf(w.s - own, fix, 1.f);
  return w;
}

// One CTA or cluster per row, in one pass over it. kPolicy: the whole row is in
// registers, and its loss and gradient follow; else the row's statistics alone,
// in as many rounds as it takes. Bound by HBM where there are many rows
// (4096 x 16000 bf16: 48 and 25 us, 39 and 19 at the copy rate), else by latency:
// with the launch of the sums 24 x 32000 fp32 takes 7.7 us, and the statistics of
// 16 x 151936 bf16 4.7.
template <typename T, bool kPolicy>
__global__ void __launch_bounds__(kRowThreadsMax) row_kernel(const RowArgs a) {
  pdl_allow_dependents();
  __shared__ RowShared sh;
  const uint32_t ctas = cluster_size(), rank = ctas == 1 ? 0u : cluster_rank();
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  pdl_wait_predecessor();
  const int64_t row = blockIdx.x / ctas;
  const Row<T> r(a.logits, row, a.ld, a.cols);
  const int64_t target = a.targets[row];
  float w = 1.f;
  if (a.weights) w = a.weights[row];
  const int warps = static_cast<int>(blockDim.x >> 5);
  const int first = (static_cast<int>(rank) * warps + static_cast<int>(threadIdx.x >> 5)) * kChunkPieces;  // the warp's chunk
  const int k0 = first + static_cast<int>(threadIdx.x & 31);
  T* g = nullptr;
  if (kPolicy && a.grad) g = static_cast<T*>(a.grad) + row * a.ld_grad;
  const bool same = same_offset(r.p, g);
  const bool leader = rank == 0 && threadIdx.x == 0;
  if (target < 0 || w == 0.f) {  // not scored: the logits are not read
    if (leader) {
      a.logp[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
      if (a.stat) a.stat[row] = make_float2(0.f, 1.f);
      if (a.coef) a.coef[row] = 0.f;
      if (kPolicy) a.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (kPolicy && g) store_zeros<T, kPieces>(r, g, same, first, k0);
    if (ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    return;
  }
  // beyond the row: no such token, everything that depends on it is NaN
  const int token = target < a.cols ? static_cast<int>(target) : kNoToken;
  const float zt = token != kNoToken ? Elem<T>::get(r.p + token) : __int_as_float(0x7fc00000);
  uint4 q[kPieces];
  MaxSum ws{-INFINITY, 0.f};
  if (kPolicy) {
    r.load(first, k0, q);
    ws = warp_stats<T>(q);
  } else {
    const int step = static_cast<int>(ctas) * warps * kChunkPieces;
    for (int k = 0; first + k < r.pieces; k += step) {
      r.load(first + k, k0 + k, q);
      ws = join(ws, warp_stats<T>(q));
    }
  }
  const MaxSum all = row_join(ws, sh, rank, ctas);
  if (!kPolicy && threadIdx.x >= 32) return;
  float rest;
  const float logp = log_prob(zt, all, &rest);
  if (!kPolicy) {
    if (leader) {
      a.logp[row] = logp;
      if (a.lse) a.lse[row] = -log_prob(0.f, all);
      if (a.stat) a.stat[row] = make_float2(all.m, all.s);
      if (a.coef) a.coef[row] = 0.f;
    }
    return;
  }
  const TokenLoss t = policy_token(logp, rest, a.old_logp[row], a.advantages[row], a.ref_logp + row, a.clip_lo, a.clip_hi, a.kl);
  if (leader) {
    a.logp[row] = logp;
    a.terms[row] = make_float4(w * (t.surrogate + a.kl * t.k3), w * t.surrogate, w * t.k3, w * t.clipped);
  }
  if (!g) return;
  const float c = w * t.slope * (a.grad_scale ? *a.grad_scale : 1.f);
  if (c == 0.f) {
    store_zeros<T, kPieces>(r, g, same, first, k0);
    return;
  }
  store_grad(r, g, same, first, k0, q, GradScale(c, all.m, all.s), token, zt);
}

// Rows of up to 32 P pieces (4 KB with P = 8), a warp each: no joins. The
// instructions that a row takes whatever its length (some 300) bound it below
// 1 KB, HBM above. 1000000 x 256 bf16 with the gradient and its sums 542 us (151 at
// the copy rate), a CTA per row 1768; 200000 x 2000 288 (236). With the logits of a
// warp's next row loaded while it works on one a fifth slower: registers.
template <typename T, bool kPolicy, int P>
__global__ void __launch_bounds__(kShortThreads) short_kernel(const RowArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  struct Scalars {
    int64_t target;
    float w, old_logp, advantage, ref_logp;
  };
  auto fetch = [&](int64_t row) {
    Scalars s{-1, 1.f, 0.f, 0.f, 0.f};
    if (row < a.rows) {
      s.target = a.targets[row];
      if (a.weights) s.w = a.weights[row];
      if (kPolicy) {
        s.old_logp = a.old_logp[row], s.advantage = a.advantages[row];
        if (a.kl != 0.f) s.ref_logp = a.ref_logp[row];
      }
    }
    return s;
  };
  constexpr int kWarps = kShortThreads / 32;
  const int lane = static_cast<int>(threadIdx.x & 31);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kWarps;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const float gs = kPolicy && a.grad_scale ? *a.grad_scale : 1.f;
  for (Scalars next = fetch(row); row < a.rows; row += stride) {
    const Scalars s = next;
    next = fetch(row + stride);
    const Row<T> r(a.logits, row, a.ld, a.cols);
    T* g = kPolicy && a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
    const bool same = same_offset(r.p, g);
    float logp = 0.f, lse = 0.f, c = 0.f, zt = 0.f;
    MaxSum all{0.f, 1.f};
    float4 terms = make_float4(0.f, 0.f, 0.f, 0.f);
    const int token = s.target < a.cols ? static_cast<int>(s.target) : kNoToken;
    uint4 q[P];
    if (s.target >= 0 && s.w != 0.f) {  // else not scored: the logits are not read
      zt = token != kNoToken ? Elem<T>::get(r.p + token) : __int_as_float(0x7fc00000);
      r.load(0, lane, q);
      all = warp_stats<T>(q);
      zt = __shfl_sync(0xffffffffu, zt, 0);  // read by now: the gradient may lie in the logits' place
      float rest;
      logp = log_prob(zt, all, &rest);
      if (!kPolicy) lse = -log_prob(0.f, all);
      if (kPolicy) {
        const TokenLoss t = policy_token(logp, rest, s.old_logp, s.advantage, &s.ref_logp, a.clip_lo, a.clip_hi, a.kl);
        terms = make_float4(s.w * (t.surrogate + a.kl * t.k3), s.w * t.surrogate, s.w * t.k3, s.w * t.clipped);
        c = s.w * t.slope * gs;
      }
    }
    if (lane == 0) {
      a.logp[row] = logp;
      if (!kPolicy && a.lse) a.lse[row] = lse;
      if (!kPolicy && a.stat) a.stat[row] = make_float2(all.m, all.s);
      if (!kPolicy && a.coef) a.coef[row] = 0.f;
      if (kPolicy) a.terms[row] = terms;
    }
    if (g) {
      if (c == 0.f) store_zeros<T, P>(r, g, same, 0, lane);
      else store_grad(r, g, same, 0, lane, q, GradScale(c, all.m, all.s), token, zt);
    }
  }
}

// The policy terms and coefficients of rows whose statistics are known, from which logp is worked out once more for
// what its rounding took off. Latency bounds it: one gathered logit per row.
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_terms_kernel(const RowArgs a) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (row >= a.rows) return;
  const float w = a.weights ? a.weights[row] : 1.f;
  float4 terms = make_float4(0.f, 0.f, 0.f, 0.f);
  const int64_t target = a.targets[row];
  if (target >= 0 && w != 0.f) {
    const float2 stat = a.stat[row];
    const float zt = target < a.cols ? Elem<T>::get(static_cast<const T*>(a.logits) + row * a.ld + target) : __int_as_float(0x7fc00000);
    float rest;
    const float logp = log_prob(zt, MaxSum{stat.x, stat.y}, &rest);
    const TokenLoss t = policy_token(logp, rest, a.old_logp[row], a.advantages[row], a.ref_logp + row, a.clip_lo, a.clip_hi, a.kl);
    terms = make_float4(w * (t.surrogate + a.kl * t.k3), w * t.surrogate, w * t.k3, w * t.clipped);
    a.coef[row] = w * t.slope * (a.grad_scale ? *a.grad_scale : 1.f);
  }
  a.terms[row] = terms;
}

// out = sum of n terms, in a fixed order, by one block.
struct Total {
  const float* terms;
  int64_t n;
  float* out;  // NULL: nothing to do
  __device__ __forceinline__ void write(WideSum* sh) const {
    WideSum s;
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s.add(terms[i]);
    const float t = block_total(s, sh);
    if (threadIdx.x == 0) *out = t;
  }
};

// Gradient of the logits from each row's statistics and coefficient, the last
// rows first (x, the part of a row, runs faster than y, the row, or kRows of them,
// each a part of the block's warps). Bound by HBM:
// 4096 x 50001 bf16 122 us alone, the copy rate. After the statistics, first rows
// first -> last rows first: 9600 x 32000 214 -> 209 us, 1600 x 32000 34 -> 31.
template <typename T, int kRows>
__global__ void __launch_bounds__(kGradThreads) grad_kernel(const RowArgs a, const Total total) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  if (total.out && blockIdx.x == 0 && blockIdx.y == 0) {
    __shared__ WideSum sh[kGradThreads / 32];
    total.write(sh);
  }
  constexpr int kWarps = kGradThreads / 32, kOfRow = kWarps / kRows;
  const int warp = static_cast<int>(threadIdx.x >> 5);
  for (int64_t row = a.rows - 1 - (static_cast<int64_t>(blockIdx.y) * kRows + warp / kOfRow); row >= 0; row -= gridDim.y * kRows) {
    const Row<T> r(a.logits, row, a.ld, a.cols);
    const int first = (static_cast<int>(blockIdx.x) * kWarps + warp % kOfRow) * 32 * kGradPieces;
    const int k0 = first + static_cast<int>(threadIdx.x & 31);
    T* g = static_cast<T*>(a.grad) + row * a.ld_grad;
    const bool same = same_offset(r.p, g);
    const float c = a.coef[row];
    if (c == 0.f) {
      store_zeros<T, kGradPieces>(r, g, same, first, k0);
      continue;
    }
    const float2 stat = a.stat[row];
    const int64_t target = a.targets[row];
    uint4 q[kGradPieces];
    r.load(first, k0, q);
    const int token = target < a.cols ? static_cast<int>(target) : kNoToken;
    // read by the thread that will write it, since the gradient may lie in the logits' place
    const float zt = holds<T, kGradPieces>(r, k0, token) ? Elem<T>::get(r.p + token) : 0.f;
    store_grad(r, g, same, first, k0, q, GradScale(c, stat.x, stat.y), token, zt);
  }
}

// One block per pair: the weighted sums of logp - ref over the two answers,
// the loss, and the coefficients of their rows. A few bytes per row: latency
// bounds it.
__global__ void __launch_bounds__(kThreads) pair_kernel(const RowArgs a, const int64_t* __restrict__ starts, float beta,
                                                        float smoothing, float inv_pairs, float* __restrict__ margins,
                                                        float* __restrict__ pair_loss) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[kThreads / 32];
  const int64_t j = blockIdx.x;
  const int64_t s0 = starts[2 * j], s1 = starts[2 * j + 1], s2 = starts[2 * j + 2];
  if (!(0 <= s0 && s0 <= s1 && s1 <= s2 && s2 <= a.rows)) {  // no such answers: NaN, and no gradient
    if (threadIdx.x == 0) margins[j] = pair_loss[j] = __int_as_float(0x7fc00000);
    return;
  }
  WideSum d;
  for (int64_t i = s0 + threadIdx.x; i < s2; i += kThreads) {
    const float w = a.weights ? a.weights[i] : 1.f;
    if (a.targets[i] < 0 || w == 0.f) continue;
    const float x = w * (a.logp[i] - a.ref_logp[i]);
    d.add(i < s1 ? x : -x);
  }
  const float x = beta * block_total(d, sh);
  // -log sigma(y) = max(-y, 0) + log(1 + exp(-|y|))
  const float e = expf(-fabsf(x)), tail = log1pf(e);
  const float sigma = x >= 0.f ? 1.f / (1.f + e) : e / (1.f + e);
  // sigma(-x) = 1 - sigma(x) without its cancellation
  const float anti = x >= 0.f ? e / (1.f + e) : 1.f / (1.f + e);
  if (threadIdx.x == 0) {
    margins[j] = x;
    pair_loss[j] = inv_pairs * ((1.f - smoothing) * (fmaxf(-x, 0.f) + tail) + smoothing * (fmaxf(x, 0.f) + tail));
  }
  if (!a.grad) return;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float slope = (smoothing * sigma - (1.f - smoothing) * anti) * beta * inv_pairs * gs;
  for (int64_t i = s0 + threadIdx.x; i < s2; i += kThreads) {
    const float w = a.weights ? a.weights[i] : 1.f;
    if (a.targets[i] < 0 || w == 0.f) continue;
    a.coef[i] = w * (i < s1 ? slope : -slope);
  }
}

constexpr int kSumThreads = 512;
constexpr int64_t kSumRows = 8192;  // of a block
__global__ void __launch_bounds__(kSumThreads) total_kernel(const Total total) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[kSumThreads / 32];
  total.write(sh);
}
// The four sums of the policy loss over the rows' terms, each in a fixed order:
// a block adds up `per` of the n terms, which lie `stride` apart, into sums, or
// (NULL) into the first of them. Latency bounds it: a block takes 5 us for 8192.
__global__ void __launch_bounds__(kSumThreads) policy_sums_kernel(float4* terms, int64_t n, int64_t stride, int64_t per, float* sums) {
  pdl_allow_dependents();
  pdl_wait_predecessor();
  __shared__ WideSum sh[4][kSumThreads / 32];
  WideSum s[4];
  const int64_t first = blockIdx.x * per, end = min(first + per, n);
  for (int64_t i = first + threadIdx.x; i < end; i += kSumThreads) {
    const float4 q = terms[i * stride];
    s[0].add(q.x), s[1].add(q.y), s[2].add(q.z), s[3].add(q.w);
  }
  if (!sums) sums = reinterpret_cast<float*>(terms + first * stride);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float t = block_total(s[k], sh[k]);  // every term has been read
    if (threadIdx.x == 0) sums[k] = t;
  }
}

// ------------------------------------------------------------------- host
meq_status fail(meq_status s, const std::string& msg) {
  meq::set_global_error(msg);
  return s;
}
meq_status launch_status(cudaError_t e, const char* fn, const char* what) {
  if (e == cudaSuccess) return MEQ_OK;
  return fail(MEQ_ERR_CUDA, std::string(fn) + ": " + what + ": " + cudaGetErrorString(e));
}
template <typename F>
meq_status guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return MEQ_ERR_OOM;
  } catch (...) {
    return MEQ_ERR_INVALID_ARG;
  }
}

int elem_bytes(int type) { return type == MEQ_F32 ? 4 : 2; }

// How a row of `cols` elements is spread over a cluster.
struct RowShape {
  int ctas, threads;
  bool held;  // the row fits into the cluster's registers
  int lanes;  // a warp holds the row, with this many pieces per lane (0: it does not)
  int sms;
};
RowShape row_shape(int64_t rows, int64_t cols, int type, int sms) {
  const int n = 16 / elem_bytes(type);
  const int64_t pieces = (cols + 2 * n - 2) / n;  // of a row that starts anywhere
  RowShape s{1, 32, true, 0, sms};
  auto need = [&](int ctas) { return (pieces + static_cast<int64_t>(ctas) * kPieces - 1) / (static_cast<int64_t>(ctas) * kPieces); };
  while (s.ctas < kMaxCluster && need(s.ctas) > kRowThreads) s.ctas *= 2;
  // few rows: more SMs to each
  while (s.ctas < kMaxCluster && rows * s.ctas * 2 <= 2 * sms && need(s.ctas) > 64) s.ctas *= 2;
  const int64_t t = (need(s.ctas) + 31) / 32 * 32;
  s.held = t <= kRowThreadsMax;
  s.threads = static_cast<int>(s.held ? t : kRowThreads);
  if (pieces <= 32 * kPieces)
    for (s.lanes = 1; pieces > 32 * s.lanes;) s.lanes *= 2;
  return s;
}

template <typename T, bool kPolicy>
cudaError_t launch_short(const RowArgs& a, const RowShape& s, cudaStream_t st) {
  constexpr int kWarps = kShortThreads / 32;
  const int64_t blocks = (a.rows + kWarps - 1) / kWarps, most = static_cast<int64_t>(s.sms) * kShortPerSm;
  const dim3 grid(static_cast<unsigned>(blocks < most ? blocks : most)), block(kShortThreads);
  if (s.lanes == 1) return launch_pdl(short_kernel<T, kPolicy, 1>, grid, block, 0, st, 1, a);
  if (s.lanes == 2) return launch_pdl(short_kernel<T, kPolicy, 2>, grid, block, 0, st, 1, a);
  if (s.lanes == 4) return launch_pdl(short_kernel<T, kPolicy, 4>, grid, block, 0, st, 1, a);
  return launch_pdl(short_kernel<T, kPolicy, 8>, grid, block, 0, st, 1, a);
}

template <bool kPolicy>
cudaError_t launch_rows_of(const RowArgs& a, int type, const RowShape& s, cudaStream_t st) {
  if (stream_suits(a.rows, a.cols, elem_bytes(type), kPolicy)) return launch_stream(a, type, kPolicy, st);
  if (s.lanes) {
    if (type == MEQ_F32) return launch_short<float, kPolicy>(a, s, st);
    if (type == MEQ_BF16) return launch_short<__nv_bfloat16, kPolicy>(a, s, st);
    return launch_short<__half, kPolicy>(a, s, st);
  }
  const dim3 grid(static_cast<unsigned>(a.rows * s.ctas)), block(s.threads);
  if (type == MEQ_F32) return launch_pdl(row_kernel<float, kPolicy>, grid, block, 0, st, s.ctas, a);
  if (type == MEQ_BF16) return launch_pdl(row_kernel<__nv_bfloat16, kPolicy>, grid, block, 0, st, s.ctas, a);
  return launch_pdl(row_kernel<__half, kPolicy>, grid, block, 0, st, s.ctas, a);
}

cudaError_t launch_terms(const RowArgs& a, int type, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.rows + kThreads - 1) / kThreads)), block(kThreads);
  if (type == MEQ_F32) return launch_pdl(policy_terms_kernel<float>, grid, block, 0, st, 1, a);
  if (type == MEQ_BF16) return launch_pdl(policy_terms_kernel<__nv_bfloat16>, grid, block, 0, st, 1, a);
  return launch_pdl(policy_terms_kernel<__half>, grid, block, 0, st, 1, a);
}

template <typename T>
cudaError_t launch_grad(const RowArgs& a, const Total& total, cudaStream_t st) {
  constexpr int kWarps = kGradThreads / 32;
  constexpr int64_t per = kGradPieces * kGradThreads;
  const int64_t pieces = (a.cols + 2 * Elem<T>::N - 2) / Elem<T>::N;
  // rows that a warp covers: as many of a block as it has warps (1000000 x 256 bf16: 900 -> 380 us)
  const int64_t rows = pieces * kWarps <= per ? kWarps : 1, blocks = (a.rows + rows - 1) / rows;
  const dim3 grid(static_cast<unsigned>((pieces + per - 1) / per), static_cast<unsigned>(blocks < 65535 ? blocks : 65535)), block(kGradThreads);
  return launch_pdl(rows == 1 ? grad_kernel<T, 1> : grad_kernel<T, kWarps>, grid, block, 0, st, 1, a, total);
}
cudaError_t launch_grad(const RowArgs& a, const Total& total, int type, cudaStream_t st) {
  if (type == MEQ_F32) return launch_grad<float>(a, total, st);
  if (type == MEQ_BF16) return launch_grad<__nv_bfloat16>(a, total, st);
  return launch_grad<__half>(a, total, st);
}

int device_sms(cudaError_t* e) {
  int dev = 0, sms = 0;
  *e = cudaGetDevice(&dev);
  if (*e == cudaSuccess) *e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// The checks that the three calls share; an empty text: fine.
std::string check_logits(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                         const float* logp) {
  if (type != MEQ_F32 && type != MEQ_BF16 && type != MEQ_F16) return "type must be a meq_dtype";
  if (rows < 0 || rows > (int64_t(1) << 27)) return "rows must be in 0..2^27";
  if (cols < 1 || cols > (int64_t(1) << 28)) return "cols must be in 1..2^28";
  if (rows > 1 && ld < cols) return "the row stride must be at least cols";
  if (ld < 0 || ld > (int64_t(1) << 40)) return "the row stride must be in 0..2^40";
  if (rows > 0 && (!logits || !targets || !logp)) return "logits, targets and logp must not be NULL";
  if (!aligned_to(logits, elem_bytes(type)) || !aligned_to(targets, 8) || !aligned_to(logp, 4))
    return "a pointer is not aligned to its type";
  return "";
}
std::string check_grad(const void* grad, int64_t ld_grad, int type, int64_t rows, int64_t cols, const float* grad_scale,
                       const float* work) {
  if (!work || !aligned_to(work, 16)) return "work must not be NULL and be 16-byte aligned";
  if (grad && rows > 1 && ld_grad < cols) return "the gradient's row stride must be at least cols";
  if (grad && (ld_grad < 0 || ld_grad > (int64_t(1) << 40))) return "the gradient's row stride must be in 0..2^40";
  if (!aligned_to(grad, elem_bytes(type)) || !aligned_to(grad_scale, 4)) return "a pointer is not aligned to its type";
  return "";
}

}  // namespace

extern "C" {

meq_status meq_token_logprobs(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                              float* logp, float* lse, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    const std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_token_logprobs: " + why);
    if (!aligned_to(lse, 4)) return fail(MEQ_ERR_INVALID_ARG, "meq_token_logprobs: a pointer is not aligned to its type");
    if (rows == 0) return MEQ_OK;
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_token_logprobs", "device attributes");
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets, a.logp = logp, a.lse = lse;
    return launch_status(launch_rows_of<false>(a, type, row_shape(rows, cols, type, sms), static_cast<cudaStream_t>(cuda_stream)),
                         "meq_token_logprobs", "launch");
  });
}

meq_status meq_debug_loss_wait(float timeout_ms, int64_t withheld_row) {
  return guarded([&]() -> meq_status {
    if (!(timeout_ms >= 0.f && timeout_ms <= 60000.f)) return fail(MEQ_ERR_INVALID_ARG, "meq_debug_loss_wait: timeout_ms must be in 0..60000");
    stream_wait(static_cast<unsigned long long>(static_cast<double>(timeout_ms) * 1e6), withheld_row);
    return MEQ_OK;
  });
}

int64_t meq_loss_work_floats(int64_t rows, int64_t pairs) { return rows < 0 || pairs < 0 ? 0 : 7 * rows + pairs + 4; }

meq_status meq_policy_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                           const float* old_logp, const float* advantages, const float* weights, const float* ref_logp,
                           float clip_low, float clip_high, float kl_coef, float* sums, float* logp, void* grad,
                           int64_t ld_grad, const float* grad_scale, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (why.empty()) why = check_grad(grad, ld_grad, type, rows, cols, grad_scale, work);
    if (why.empty() && rows > 0 && (!old_logp || !advantages)) why = "old_logp and advantages must not be NULL";
    if (why.empty() && (!sums || !aligned_to(sums, 4))) why = "sums must not be NULL";
    if (why.empty() && !(clip_low >= 0.f && clip_low <= 1.f && clip_high >= 0.f && std::isfinite(clip_high)))
      why = "clip_low must be in 0..1 and clip_high finite and >= 0";
    if (why.empty() && !(kl_coef >= 0.f && std::isfinite(kl_coef))) why = "kl_coef must be finite and >= 0";
    if (why.empty() && kl_coef > 0.f && rows > 0 && !ref_logp) why = "a KL term needs ref_logp";
    if (why.empty() && !(aligned_to(old_logp, 4) && aligned_to(advantages, 4) && aligned_to(weights, 4) && aligned_to(ref_logp, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_policy_loss: " + why);
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets;
    a.old_logp = old_logp, a.advantages = advantages, a.weights = weights, a.ref_logp = ref_logp;
    a.clip_lo = 1.f - clip_low, a.clip_hi = 1.f + clip_high, a.kl = kl_coef, a.grad_scale = grad_scale;
    a.logp = logp, a.terms = reinterpret_cast<float4*>(work), a.grad = grad, a.ld_grad = ld_grad;
    if (rows > 0) {
      const RowShape s = row_shape(rows, cols, type, sms);
      if (s.held || stream_suits(rows, cols, elem_bytes(type), true)) {
        e = launch_rows_of<true>(a, type, s, st);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "launch");
      } else {
        a.stat = reinterpret_cast<float2*>(work + 4 * rows), a.coef = work + 6 * rows;
        e = launch_rows_of<false>(a, type, s, st);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "statistics launch");
        e = launch_terms(a, type, st);
        if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "terms launch");
        if (grad) {
          e = launch_grad(a, Total{}, type, st);
          if (e != cudaSuccess) return launch_status(e, "meq_policy_loss", "gradient launch");
        }
      }
    }
    float4* terms = reinterpret_cast<float4*>(work);
    const int64_t blocks = (rows + kSumRows - 1) / kSumRows;
    if (blocks <= 1) {
      e = launch_pdl(policy_sums_kernel, dim3(1), dim3(kSumThreads), 0, st, 1, terms, rows, int64_t(1), rows, sums);
    } else {
      e = launch_pdl(policy_sums_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kSumThreads), 0, st, 1, terms, rows, int64_t(1), kSumRows,
                     static_cast<float*>(nullptr));
      if (e == cudaSuccess) e = launch_pdl(policy_sums_kernel, dim3(1), dim3(kSumThreads), 0, st, 1, terms, blocks, kSumRows, blocks, sums);
    }
    return launch_status(e, "meq_policy_loss", "sum launch");
  });
}

meq_status meq_preference_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                               const int64_t* starts, int64_t pairs, const float* ref_logp, const float* weights, float beta,
                               float label_smoothing, float* loss, float* margins, float* logp, void* grad, int64_t ld_grad,
                               const float* grad_scale, float* work, void* cuda_stream) {
  return guarded([&]() -> meq_status {
    std::string why = check_logits(logits, type, rows, cols, ld, targets, logp);
    if (why.empty()) why = check_grad(grad, ld_grad, type, rows, cols, grad_scale, work);
    if (why.empty() && (pairs < 1 || pairs > (int64_t(1) << 27))) why = "pairs must be in 1..2^27";
    if (why.empty() && (!starts || !loss || !margins || (rows > 0 && !ref_logp))) why = "starts, ref_logp, loss and margins must not be NULL";
    if (why.empty() && !(std::isfinite(beta) && beta > 0.f)) why = "beta must be finite and > 0";
    if (why.empty() && !(label_smoothing >= 0.f && label_smoothing <= 1.f)) why = "label_smoothing must be in 0..1";
    if (why.empty() && !(aligned_to(starts, 8) && aligned_to(ref_logp, 4) && aligned_to(weights, 4) && aligned_to(loss, 4) && aligned_to(margins, 4)))
      why = "a pointer is not aligned to its type";
    if (!why.empty()) return fail(MEQ_ERR_INVALID_ARG, "meq_preference_loss: " + why);
    cudaError_t e;
    const int sms = device_sms(&e);
    if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "device attributes");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    RowArgs a{};
    a.logits = logits, a.rows = rows, a.cols = cols, a.ld = ld, a.targets = targets, a.weights = weights, a.ref_logp = ref_logp;
    a.grad_scale = grad_scale, a.logp = logp, a.stat = reinterpret_cast<float2*>(work + 4 * rows), a.coef = work + 6 * rows;
    a.grad = grad, a.ld_grad = ld_grad;
    float* pair_loss = work + 7 * rows;
    if (rows > 0) {
      e = launch_rows_of<false>(a, type, row_shape(rows, cols, type, sms), st);
      if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "statistics launch");
    }
    e = launch_pdl(pair_kernel, dim3(static_cast<unsigned>(pairs)), dim3(kThreads), 0, st, 1, a, starts, beta, label_smoothing,
                   static_cast<float>(1.0 / static_cast<double>(pairs)), margins, pair_loss);
    if (e != cudaSuccess) return launch_status(e, "meq_preference_loss", "pair launch");
    const Total total{pair_loss, pairs, loss};
    if (grad && rows > 0)
      return launch_status(launch_grad(a, total, type, st), "meq_preference_loss", "gradient launch");
    return launch_status(launch_pdl(total_kernel, dim3(1), dim3(kSumThreads), 0, st, 1, total), "meq_preference_loss", "sum launch");
  });
}

}  // extern "C"

/*
 * meq.h -- C ABI of the GB300 (sm_103a) MeqMuon optimizer step for 2D
 * hidden-layer weights.
 *
 * The step follows the paper "MeqMuon: Matrix-Equilibrating Muon for LLM
 * Pretraining", Algorithm 1 (hidden-weight branch), for every matrix W_i:
 *
 *   B_t   = mu B_{t-1} + G_t                                   Eq. (10)
 *   U_t   = NS_K(B_t)  (X_0 = B/||B||_F;
 *           X_{k+1} = a X_k + (b A_k + c A_k^2) X_k, A_k = X_k X_k^T)  Eq. (5)
 *   r_i = ||U_{i,:}||/sqrt(n), c_j = ||U_{:,j}||/sqrt(m)       Eq. (7)
 *   gamma = std/mean over entries > eps                        Eq. (8)
 *   U~  = diag(r^-1) U  if gamma_r >= gamma_c, else U diag(c^-1)  Eqs. (9), (11)
 *   W  <- (1 - lr*wd) W - rho*lr*U~                            Eq. (14)
 *
 * Everything runs in the library's own CUDA kernels, asynchronously on the
 * caller's stream. Newton-Schulz runs on the tensor cores (tcgen05, TMA, TMEM)
 * with 16-bit operands and fp32 accumulation; all other arithmetic is fp32.
 *
 * Conventions shared by every call:
 *   - Matrices are fp32, row-major, contiguous, rows = output features and
 *     columns = input features (the PyTorch layout the paper uses, Section 3.1).
 *   - Device pointers must be 16-byte aligned.
 *   - A meq_state is not thread-safe: one host thread drives it at a time.
 *   - Validation errors are returned synchronously and nothing is enqueued.
 *     Errors raised on the device (a bounded wait that expired) are reported
 *     by the next meq_sync() as MEQ_ERR_TIMEOUT / MEQ_ERR_CUDA.
 */
#ifndef MEQ_H
#define MEQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MEQ_OK = 0,
  MEQ_ERR_INVALID_ARG = 1,   /* null pointer, bad size, misaligned pointer, shape list differs from init */
  MEQ_ERR_OOM = 2,           /* device allocation failed or the workspace limit was exceeded */
  MEQ_ERR_CUDA = 3,          /* a CUDA runtime call failed (see meq_last_error) */
  MEQ_ERR_NONFINITE = 4,     /* a step's momentum had a non-finite norm (reported by meq_sync) */
  MEQ_ERR_TIMEOUT = 5,       /* a device-side bounded wait expired; the kernel returned early */
  MEQ_ERR_UNSUPPORTED = 6,   /* no sm_103a device, or a size beyond the library's limits */
  MEQ_ERR_CORRUPTED = 7      /* meq_check_canaries found a workspace guard band overwritten */
} meq_status;

/* One matrix: rows = out features (m), cols = in features (n). */
typedef struct {
  int64_t rows;
  int64_t cols;
} meq_shape;

/* Options fixed at init. meq_default_options() fills the paper's values. */
typedef struct {
  float rho;              /* RMS alignment coefficient, Eq. (14); 0.2 (Section 4) */
  int ns_steps;           /* K of Eq. (5); 5 (Sections 2 and 4); 1..32 */
  float ns_a, ns_b, ns_c; /* (3.4445, -4.7750, 2.0315), Section 2 */
  int nesterov;           /* 0: NS input B_t (Eq. (10), Algorithm 1);
                             1: NS input G_t + mu B_t (Nesterov look-ahead, Section 4) */
  uint32_t ns_fp16_mask;  /* bit k set: NS iteration k uses fp16 operands, else bf16.
                             Default 0xFFFFFFFF (all fp16; same tensor-core rate as bf16,
                             three more mantissa bits). 0 = all bf16. */
  float tie_atol;         /* Eq. (11) chooses row when gamma_r >= gamma_c - tie_atol; 1e-6 */
  int use_graph;          /* 1: the step's kernels are replayed from a CUDA graph (default) */
  int64_t workspace_limit_bytes; /* 0 = no limit; else init fails with MEQ_ERR_OOM above it */
  float wait_timeout_ms;  /* bound of every device-side spin wait; default 4000. An NS kernel's
                             MMA thread starts waiting for its first operands while the kernel
                             before it may still run, so the bound must exceed the longest kernel
                             of a step (about 20 ms per NS product at Llama-7B-class sizes) */
  int ns_cta_pair;        /* 1 (default): NS GEMMs run on CTA pairs (tcgen05 cta_group::2,
                             256 x 256 tiles on two SMs); 0: one CTA per 128 x 256 tile */
  int ns_x0_fused;        /* 1 (default): the momentum pass also writes X_0, unnormalised in
                             bf16, and the first NS products apply 1/||B||_F; iteration 0
                             then runs its X and P operands in bf16. 0: a separate pass
                             writes the normalised X_0 in the format ns_fp16_mask gives it. */
  int update_rule;        /* meq_update_rule; default MEQ_RULE_MEQMUON */
  int debug_canaries;     /* 1: guard bands of a fixed byte pattern surround every workspace
                             buffer (meq_check_canaries); default 0 */
  int debug_skip_load;    /* 1 (tests only): in every step's first NS launch, the leader
                             CTA of the first CTA pair arms its first operand stage but
                             does not load its half, so that stage never completes: the
                             MMA issuer's bounded wait expires, every role of the launch
                             stops and drains, and meq_sync reports MEQ_ERR_TIMEOUT (the
                             results of that step are not meaningful). Requires
                             ns_cta_pair = 1. Default 0. */
} meq_options;

/* Update applied to the hidden 2D weights after momentum and Newton-Schulz. */
typedef enum {
  MEQ_RULE_MEQMUON = 0, /* Eq. (11) equilibration, then Eq. (14) (Algorithm 1) */
  MEQ_RULE_MUON = 1     /* Muon with decoupled weight decay and RMS alignment, Eq. (6)
                           (the comparison baseline of Section 4): W <- (1 - lr wd) W
                           - lr rho sqrt(max(m, n)) U, no equilibration. Every entry must
                           be MEQ_KIND_HIDDEN (that baseline updates the others with
                           AdamW: a meq_adamw state of their own). */
} meq_update_rule;

/* Parameter type, selecting the branch of Algorithm 1 applied to it. */
typedef enum {
  MEQ_KIND_HIDDEN = 0,       /* 2D weight in a hidden layer: NS, then Eq. (11) (default) */
  MEQ_KIND_REMAINING_2D = 1, /* token embedding / LM head: N_c(N_r(B_t)), Eq. (12) */
  MEQ_KIND_VECTOR = 2        /* 1D parameter, given as shape (1, d): B_t / (||B_t||/sqrt(d)), Eq. (13) */
} meq_kind;

typedef struct meq_state meq_state; /* opaque */

void meq_default_options(meq_options* opt);

/* Bytes the state would allocate for this shape list, computed on the host
 * without touching the GPU. persistent = momentum buffers (4 bytes per
 * element: the only state MeqMuon keeps, Section 4 "Memory overhead");
 * workspace = transient NS / statistics buffers. Either output may be NULL. */
meq_status meq_state_bytes(const meq_shape* shapes, int n, const meq_options* opt,
                           size_t* persistent_bytes, size_t* workspace_bytes);

/* As meq_state_bytes, with a parameter type per entry (kinds may be NULL:
 * all MEQ_KIND_HIDDEN). MEQ_KIND_VECTOR entries must have rows == 1. */
meq_status meq_state_bytes_kinds(const meq_shape* shapes, const int* kinds, int n, const meq_options* opt,
                                 size_t* persistent_bytes, size_t* workspace_bytes);

/* Create the state for n matrices: zeroed momentum (B_{-1} = 0, Algorithm 1)
 * and the workspace, on the current CUDA device. opt may be NULL (defaults).
 * cuda_stream (cudaStream_t, may be NULL) orders the zero-fill. The shape
 * list is copied. On success *out owns device memory until meq_free.
 * Entries are updated independently: the launches are planned for the whole
 * list, but every result of an entry is the same bit for bit whatever else
 * the list holds (so a list split over several states gives what one gives). */
meq_status meq_init_state(const meq_shape* shapes, int n, const meq_options* opt,
                          void* cuda_stream, meq_state** out);

/* As meq_init_state, with a parameter type (meq_kind) per entry, so one state
 * runs Algorithm 1 over every trainable parameter of a model: hidden 2D
 * weights, the other 2D parameters, and vectors (shape (1, d)).
 * kinds is copied; NULL means all MEQ_KIND_HIDDEN. */
meq_status meq_init_state_kinds(const meq_shape* shapes, const int* kinds, int n,
                                const meq_options* opt, void* cuda_stream, meq_state** out);

/* One MeqMuon step over all n matrices (Algorithm 1, hidden branch).
 *   params[i]: device fp32 W_i (rows x cols), updated in place.
 *   grads[i] : device fp32 G_i, read only.
 *   shapes/n : must equal the list given to meq_init_state.
 *   lr = eta_t (the caller applies warm-up / decay), momentum = mu,
 *   weight_decay = lambda, eps = delta of Section 3.1 (1e-7).
 * All work is enqueued on cuda_stream (cudaStream_t; NULL = legacy default
 * stream) with no host synchronisation. params/grads must stay valid until
 * the enqueued work has run. */
meq_status meq_step(float* const* params, const float* const* grads, meq_state* st,
                    const meq_shape* shapes, int n, float lr, float momentum,
                    float weight_decay, float eps, void* cuda_stream);

/* The same step in two calls, split before the parameter update, so that a
 * caller can overlap work on the parameters of the previous step (a copy
 * to the host, an all-gather) with this step's momentum, Newton-Schulz and
 * statistics, which do not touch the parameters:
 *   meq_step_prepare: Eq. (10), Eq. (5) and the statistics of Eqs. (7)-(9)
 *     and (11) (Algorithm 1 up to the update), for the gradients and scalars
 *     given (the arguments of meq_step without params);
 *   meq_step_apply: the update (Eq. (14); Eqs. (12) and (13) for the other
 *     kinds) of params with the scalars of the pending prepare.
 * meq_step(params, grads, ...) equals meq_step_prepare(grads, ...) then
 * meq_step_apply(params, ...), bit for bit. Each call enqueues on its
 * cuda_stream; the apply must be ordered after its prepare and before the
 * next prepare (for example, one stream, with a cudaStreamWaitEvent on the
 * caller's copy before the apply). A second prepare before the apply, an
 * apply without a prepare, or meq_step while a prepare is pending returns
 * MEQ_ERR_INVALID_ARG. With use_graph, each part replays its own graph. */
meq_status meq_step_prepare(const float* const* grads, meq_state* st, const meq_shape* shapes, int n,
                            float lr, float momentum, float weight_decay, float eps, void* cuda_stream);
meq_status meq_step_apply(float* const* params, meq_state* st, void* cuda_stream);

/* Wait for the state's enqueued work and report device-side errors
 * (MEQ_ERR_TIMEOUT for an expired bounded wait, MEQ_ERR_CUDA otherwise), then
 * MEQ_ERR_NONFINITE if, in a step since the last meq_sync, the momentum of
 * some entry had a NaN or infinite sum of squares (a non-finite gradient, or
 * a momentum already non-finite); meq_last_error names the first such entry.
 * Each report clears the condition. Such an entry's momentum and parameters
 * take the non-finite values (no step is skipped); every other entry's step
 * is unaffected, since entries are updated independently. */
meq_status meq_sync(meq_state* st);

/* Release all device memory of the state (synchronises first). NULL is a no-op. */
meq_status meq_free(meq_state* st);

/* Human-readable text of the last error of st; with st NULL, of the last
 * failed call that this thread made without a state (meq_init_state[_kinds],
 * meq_state_bytes[_kinds], meq_ns_cv_trajectory, meq_row_col_stats_noalloc,
 * meq_adamw_init, meq_adamw_state_bytes, the loss calls).
 * Valid until its next such call. */
const char* meq_last_error(const meq_state* st);
const char* meq_status_string(meq_status s);

/* ---- inspection and checkpointing (synchronise the state first) ---------- */

/* Copy momentum B_i (rows x cols fp32) to dst (host or device memory). */
meq_status meq_read_momentum(meq_state* st, int i, float* dst);
/* Overwrite momentum B_i from src (host or device), e.g. to resume. */
meq_status meq_write_momentum(meq_state* st, int i, const float* src);
/* Copy the last step's Newton-Schulz output U_i (rows x cols fp32, before
 * equilibration) to dst (host or device). Hidden weights only. U is held on
 * the device in fp16 (scaled by 2^14, so every entry above 4e-9 keeps 11
 * significant bits); the values returned are those fp16 values, from which
 * the row and column statistics are taken and which the update applies. */
meq_status meq_read_ns_output(meq_state* st, int i, float* dst);
/* Copy the normalised update U~_i of the last step (rows x cols fp32) to
 * dst (host or device): the matrix that step applied as
 * W <- (1 - lr wd) W - rho lr U~ (Eq. (14)). Hidden weight: diag(r^-1) U or
 * U diag(c^-1) (Eqs. (9), (11); rows or columns with RMS <= eps scaled by 0),
 * or sqrt(max(m, n)) U under MEQ_RULE_MUON (Eq. (6)); remaining 2D
 * parameter: N_c(N_r(B_t)) (Eq. (12)); vector: B_t / RMS(B_t) (Eq. (13)).
 * Computed by a kernel on the state's device (whichever device is current;
 * the current device is restored) from the operands and scale factors of
 * the update kernel; a host dst goes through the state's own scratch (hidden
 * weights) or a temporary device buffer of the same size (MEQ_ERR_OOM if that
 * allocation fails). Synchronises the state's stream. */
meq_status meq_read_update(meq_state* st, int i, float* dst);
/* Last step's statistics of entry i. Hidden weight: r (rows floats), c (cols
 * floats) of Eq. (7) for U, gamma_r, gamma_c of Eq. (8) and the direction of
 * Eq. (11) (0 = row, 1 = column; 4 under MEQ_RULE_MUON, whose update is
 * the uniform sqrt(max(m, n)) U of Eq. (6) while r, c and the CVs still
 * describe U). Remaining 2D parameter: r = row RMS of B_t, c = column RMS
 * of N_r(B_t), their CVs, direction 2. Vector: r[0] = RMS of B_t, gammas 0,
 * direction 3. Any output may be NULL; r and c are host or device memory. */
meq_status meq_read_stats(meq_state* st, int i, float* r, float* c,
                          double* gamma_r, double* gamma_c, int* direction);
/* How often Eq. (11) chose row-wise (*rows) and column-wise (*cols)
 * normalisation for hidden weight i since the state was created or the
 * counts were last reset (both 0 for other entries and under MEQ_RULE_MUON).
 * The counts are kept on the device by the statistics kernel. */
meq_status meq_read_direction_counts(meq_state* st, int i, int64_t* rows, int64_t* cols);
/* Zero every entry's direction counts (enqueued on the state's stream). */
meq_status meq_reset_direction_counts(meq_state* st);

/* ---- diagnostics -------------------------------------------------------- */

/* With debug_canaries set at init: synchronise the state's stream and check
 * that every guard band still holds its pattern. MEQ_OK, or
 * MEQ_ERR_CORRUPTED with *bad_offset (may be NULL) = the arena offset of the
 * first changed byte (-1 otherwise); MEQ_ERR_INVALID_ARG without guards. */
meq_status meq_check_canaries(meq_state* st, int64_t* bad_offset);
/* Number of guard bands (0 without debug_canaries). */
int meq_canary_count(const meq_state* st);
/* Test hook: overwrite one byte of guard band `index` from the host
 * (cudaMemset), so that tests can check meq_check_canaries. */
meq_status meq_debug_corrupt_canary(meq_state* st, int index);

/* Row / column CV trajectory of the Newton-Schulz iterates (Section 3.1
 * replays Eq. (5) on saved pre-NS matrices this way): gamma_r[k] and
 * gamma_c[k] are the Eq. (8) CVs (over entries > eps) of the row and column
 * RMS (Eq. (7)) of X_k, k = 0..steps, computed by this library's CUDA path
 * with the NS options of opt (NULL: defaults; its ns_steps and update_rule
 * are ignored). k = 0 is X_0 = h / ||h||_F: its RMS values, like those of
 * every later iterate, are compared with eps after the normalisation. h:
 * device fp32, rows x cols row-major, 16-byte aligned, read only. gamma_r,
 * gamma_c: host arrays of steps + 1 doubles. steps: 0..32. Synchronous;
 * allocates and frees its own device scratch (the statistics' partial sums
 * and one optimizer state), so concurrent calls do not share memory;
 * every shape meq_init_state accepts is accepted. Errors:
 * MEQ_ERR_INVALID_ARG (NULL, misaligned, bad sizes), MEQ_ERR_OOM, or the
 * error of the step it runs (text in meq_last_error(NULL)). */
meq_status meq_ns_cv_trajectory(const float* h, int64_t rows, int64_t cols, int steps, float eps,
                                const meq_options* opt, double* gamma_r, double* gamma_c, void* cuda_stream);
/* Number of kernels one meq_step launches (for launch accounting), and how
 * many of them are Newton-Schulz GEMM launches. */
int meq_kernels_per_step(const meq_state* st);
int meq_ns_gemm_launches_per_step(const meq_state* st);
/* Columns of the output tiles of the i-th of those launches: 256, or 64 where
 * the launch has few tiles (0: no such launch). For tests and profiles. */
int meq_ns_gemm_tile_columns(const meq_state* st, int i);
/* Floating-point operations of those products (Eq. (5) as written), the
 * symmetric ones counted as one triangle. */
double meq_ns_flops_per_step(const meq_state* st);

/* Per-phase timing with CUDA events on the launch stream. While enabled,
 * meq_step runs the same kernels with an event recorded between phases:
 * with use_graph, by replaying a second graph that holds event-record nodes
 * between the phases, then waiting for the stream and adding up that step's
 * phase times (so profiled steps are not pipelined with the host); without
 * use_graph, by launching directly. meq_read_profile synchronises and returns
 * the summed milliseconds of each phase since profiling was enabled:
 *   phase_ms[0] momentum update + norms (all kinds), [1] X_0 cast,
 *   [2] all NS GEMMs, [3] statistics + direction / scales, [4] apply;
 *   *steps = profiled steps. */
meq_status meq_set_profiling(meq_state* st, int enable);
meq_status meq_read_profile(meq_state* st, double* phase_ms /* 5 */, int64_t* steps);

/* Failure-path self test of the device-side bounded waits: launches one
 * kernel that spins on a flag nothing ever sets, with the given limit
 * (0 < timeout_ms <= 10000), then synchronises. The kernel gives up when the
 * limit expires, records the timeout and returns, so the expected result is
 * MEQ_ERR_TIMEOUT with the context still usable. The paper has no
 * counterpart; this exists to test error reporting without faulting a GPU. */
meq_status meq_debug_wait_selftest(meq_state* st, float timeout_ms);

/* ---- allocation-free statistics ------------------------------------------
 * The paper has no counterpart to this entry point; it exists for callers
 * that cannot call cudaMalloc (code running inside a framework that owns all
 * device memory through its own pool, or a latency-critical path that must
 * not allocate after start-up, since cudaMalloc may synchronise the device).
 *
 * meq_row_col_stats_noalloc computes, for one fp32 row-major matrix U
 * (rows x cols, device memory, read only), the statistics step of the
 * optimizer: r (rows floats) and c (cols floats) of Eq. (7), gammas[0] =
 * gamma_r and gammas[1] = gamma_c of Eq. (8) over entries > eps, and
 * *direction of Eq. (11) (0 = row, 1 = column; row when gamma_r >= gamma_c -
 * tie_atol). All outputs are caller-provided device memory. The definitions
 * and precision (fp32 sums of squares and two-pass fp32 CVs) are those of
 * meq_step's statistics, so results agree with meq_read_stats for the same U
 * up to fp32 summation order.
 *
 * It allocates nothing. Its scratch is a fixed 8 MiB __device__ array inside
 * the library, held by every GPU that loads the library until the process
 * exits. A matrix fits when rows * ceil(cols / 1024) + ceil(rows / 32) * cols
 * <= 2,097,152 floats (e.g. 4096 x 11008 and 11008 x 4096, but not 8192 x
 * 8192); larger ones, NULL pointers or
 * non-positive sizes return MEQ_ERR_INVALID_ARG before anything is enqueued
 * and before any CUDA call; meq_last_error(NULL) then says why.
 * The first call on a device looks up the array's device address (once per
 * device, with that device current); make that first call before any CUDA
 * stream capture. Every call shares the one array and overwrites all of the
 * scratch it reads, so nothing needs clearing between calls, but calls whose
 * kernels overlap on the GPU (different streams without ordering) race on
 * it. Work is enqueued on cuda_stream (cudaStream_t, NULL = legacy stream)
 * as three kernel launches; MEQ_ERR_CUDA reports a failed launch or address
 * lookup of this call (its own status, with the CUDA error text in
 * meq_last_error(NULL)). */
meq_status meq_row_col_stats_noalloc(const float* U, int64_t rows, int64_t cols, float eps,
                                     float tie_atol, float* r, float* c, double* gammas,
                                     int* direction, void* cuda_stream);

/* ---- AdamW over many tensors ----------------------------------------------
 * AdamW for what MeqMuon does not step (embedding, head, norm weights under
 * the comparison rule of Eq. (6)) or for a whole model. For every element of
 * entry i at step t, with g' = s g:
 *
 *   m <- beta1 m + (1 - beta1) g'         v <- beta2 v + (1 - beta2) g'^2
 *   p <- (1 - lr wd decay_i) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 *
 * in fp32, whatever the types of p and g (16-bit gradients are widened, a bf16
 * parameter is rounded to nearest once, at the end). One launch per 256
 * entries; no host synchronisation and no copy, so a step can be captured into
 * a CUDA graph (the scalars and pointers of the call are then fixed).
 *
 * The moments are fp32, or 8-bit codes with one fp32 scale per 256 consecutive
 * elements for each of m and r = sqrt(v), the largest |m| and r among them:
 * m = S_m sign(q) (q / 127)^2 with q in -127..127, r = S_r (q / 255)^2 with q in
 * 0..255, rounded to the nearest code (r > 0 never to 0). The update of a step
 * uses the moments as computed, before they are rounded. A block with a
 * non-finite moment has a NaN scale; one whose largest value is below 2^-126 is
 * held as zero. Entries are independent: what an entry becomes does not depend
 * on the others of the list. Each entry's moments start at a multiple of 256
 * elements of the state's arrays, in the order of the list.
 *
 * Pointers need the alignment of their element type only; entries whose
 * tensors are all 16-byte aligned move in wide accesses. */
typedef enum { MEQ_F32 = 0, MEQ_BF16 = 1, MEQ_F16 = 2 } meq_dtype;

typedef struct {
  double beta1, beta2; /* 0.9, 0.999; in [0, 1) */
  double eps;          /* 1e-8; >= 2^-126 */
  int state_bits;      /* 32 (default) or 8 */
  int param_type;      /* MEQ_F32 (default) or MEQ_BF16 */
  int grad_type;       /* a meq_dtype; default MEQ_F32 */
} meq_adamw_options;

/* Opaque. Like a meq_state, one host thread drives it at a time, and its calls
 * follow one another in the order of the streams that they are given: use one,
 * or order them with events. meq_adamw_steps, _set_steps, _sync and _free wait
 * for the stream of the last call; once a call has been captured into a graph,
 * for the whole device, since replays may run on any stream. */
typedef struct meq_adamw meq_adamw;

void meq_adamw_default_options(meq_adamw_options* opt);
/* Bytes of the moments (with their scales) and of everything else the state
 * would allocate, computed on the host. Either output may be NULL. */
meq_status meq_adamw_state_bytes(const meq_shape* shapes, int n, const meq_adamw_options* opt,
                                 size_t* persistent_bytes, size_t* workspace_bytes);
/* State for n entries on the current device, moments and step count zero.
 * decay[i] >= 0 multiplies the weight decay of entry i (NULL: 1 for all; 0 for
 * norm weights and biases); opt may be NULL. Shapes have meq_init_state's
 * limits (2^20 rows and columns, 2^34 elements). Otherwise only their element
 * counts matter: a longer flat buffer may be given as any rows x cols with its
 * count, or as several entries. */
meq_status meq_adamw_init(const meq_shape* shapes, const float* decay, int n, const meq_adamw_options* opt,
                          void* cuda_stream, meq_adamw** out);
/* out[0] = the Euclidean norm of all gradients together, out[1] = the
 * coefficient that brings it to at most max_norm (1 if it is there; NaN if the
 * sum of squares is not finite in fp32, as with a gradient that is not or a norm
 * from 1.8e19 on). out: device, two floats. max_norm > 0, may be infinite. Sums
 * of squares: fp32 per thread, then compensated, in a fixed order; gradients
 * below some 1e-22 may not count. */
meq_status meq_adamw_grad_norm(const void* const* grads, meq_adamw* st, float max_norm, float* out, void* cuda_stream);
/* One step. params (updated in place) and grads: device, contiguous, of the
 * state's types. copies: NULL, or per entry a device bf16 tensor of its size
 * that receives the updated parameter rounded to nearest. grad_scale: NULL
 * (s = 1), or a device float s: a clipping coefficient (out + 1 of
 * meq_adamw_grad_norm), the inverse of a loss scale, or both. If s is not
 * finite the step is skipped on the device: parameters, moments and step count
 * stay as they are, and meq_adamw_sync says so. */
meq_status meq_adamw_step(void* const* params, const void* const* grads, void* const* copies, meq_adamw* st, float lr,
                          float weight_decay, const float* grad_scale, void* cuda_stream);
/* The state's own arrays (device), valid until meq_adamw_free, to checkpoint
 * and resume exactly: m and v (fp32), or the codes of m (int8) and r (uint8)
 * with their scales (else NULL); *elements = their length, entries padded to
 * multiples of 256 (scales: a 256th of it). The padding holds zeros and has to.
 * Any output may be NULL. */
meq_status meq_adamw_state_ptrs(meq_adamw* st, void** m, void** v, float** m_scale, float** v_scale, int64_t* elements);
/* The values of m and v, whichever way they are held, into device fp32 arrays
 * of *elements each, laid out as the state's (16-byte aligned; either may be
 * NULL). */
meq_status meq_adamw_read_values(meq_adamw* st, float* m, float* v, void* cuda_stream);
/* Number of steps done (waits for the state's work), and its overwriting, to
 * resume. Skipped steps do not count. */
meq_status meq_adamw_steps(meq_adamw* st, int64_t* steps);
meq_status meq_adamw_set_steps(meq_adamw* st, int64_t steps);
/* Wait for the state's work; then MEQ_ERR_NONFINITE if since the last sync a
 * step was skipped or left a non-finite moment (meq_adamw_last_error names the
 * entry; such a step is not skipped). Each report clears the condition. */
meq_status meq_adamw_sync(meq_adamw* st);
/* Releases the state (waits for its work first). NULL is a no-op. */
meq_status meq_adamw_free(meq_adamw* st);
const char* meq_adamw_last_error(const meq_adamw* st);

/* ---- losses on token log-probabilities --------------------------------------
 * The losses of fine-tuning with a policy or with preferences, from logits z
 * (rows x cols, one row per token) and one target token t_i per row:
 *
 *   logp_i = z_{i,t_i} - log sum_j exp(z_ij)
 *   dL/dz_ij = c_i ([j = t_i] - softmax_j(z_i)),  c_i = grad_scale dL/dlogp_i
 *
 * logits: device, of meq_dtype `type`, consecutive columns, rows `ld` elements
 *   apart (ld >= cols; rows may start at any element). -inf masks a token; a
 *   row with a NaN or +inf, or with -inf alone (whose lse is -inf), gives NaN.
 * targets: device int64. A negative target marks a row that is not scored: its
 *   logits are not read, its logp is 0, its gradient zero. A target >= cols
 *   gives NaN. In the losses a weight of 0 leaves a row out in the same way.
 * grad: NULL, or device memory of the logits' type for dL/dz, rows ld_grad
 *   elements apart, every row written, rounded to nearest once. It may be the
 *   logits themselves (same pointer, ld_grad = ld), else it must not overlap
 *   them. Fastest where grad and logits lie at the same offset within 16 bytes
 *   in every row.
 * grad_scale: NULL (1), or a device float that multiplies the gradient: the
 *   incoming gradient of the loss, a loss scale.
 * work: device scratch of meq_loss_work_floats floats, 16-byte aligned, free
 *   again when the enqueued kernels have run.
 * Softmax statistics and all scalars are fp32, sums over rows compensated, all
 * in fixed orders: results repeat bit for bit. A kernel's own waits are bounded
 * (4 s, and time that the context is switched out does not end one alone): a
 * thread block that gives up writes NaN as every result of all its rows, so the
 * sums become NaN too. Nothing is allocated, and the calls may come from several
 * threads. rows may be 0. Limits: rows <= 2^27,
 * cols <= 2^28. */

/* logp (rows floats) and, if lse is not NULL, log sum_j exp(z_ij) (0 for rows
 * that are not scored). */
meq_status meq_token_logprobs(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                              float* logp, float* lse, void* cuda_stream);

/* Diagnostic, for the calling thread's next loss calls: the limit of the
 * kernels' waits (0: the usual 4 s) and a row whose data never arrives where rows
 * are streamed through shared memory (-1: none), so that a wait runs out. */
meq_status meq_debug_loss_wait(float timeout_ms, int64_t withheld_row);

/* Floats of `work` for a loss over rows tokens and (meq_preference_loss) pairs
 * pairs (0: meq_policy_loss). Host only. */
int64_t meq_loss_work_floats(int64_t rows, int64_t pairs);

/* The clipped policy loss with a KL term. With r = exp(logp - old_logp),
 * A = advantages, d = ref_logp - logp (logp before it is rounded to fp32, so r of
 * one's own logp is 1 but for that rounding, and a clip_low or clip_high of 0
 * takes such a row for clipped):
 *
 *   L = sum_i w_i (s_i + kl_coef k_i)
 *   s = -min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A),  k = exp(d) - d - 1
 *
 * weights: w (NULL: 1 for all), e.g. the answer's mask over its length.
 * ref_logp is read where kl_coef > 0 only. old_logp, advantages, weights,
 * ref_logp: device, rows floats. sums: device, 4 floats: L, sum w s, sum w k,
 * and the weight of the rows whose ratio is clipped. logp: device, rows
 * floats, out. clip_low in 0..1; clip_high, kl_coef >= 0. */
meq_status meq_policy_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                           const float* old_logp, const float* advantages, const float* weights, const float* ref_logp,
                           float clip_low, float clip_high, float kl_coef, float* sums, float* logp, void* grad,
                           int64_t ld_grad, const float* grad_scale, float* work, void* cuda_stream);

/* The paired preference loss: rows starts[2j] .. starts[2j+1] - 1 are the
 * preferred answer of pair j, starts[2j+1] .. starts[2j+2] - 1 the other.
 *
 *   x_j = beta (sum_preferred w (logp - ref_logp) - sum_other w (logp - ref_logp))
 *   L = mean_j (-(1 - e) log sigma(x_j) - e log sigma(-x_j)),  e = label_smoothing
 *
 * starts: device, 2 pairs + 1 int64, not decreasing, within 0..rows (an answer
 * may be empty; a pair whose starts are not so gives NaN, itself no gradient,
 * and rows that pairs on both sides of it share get either's).
 * ref_logp per token, as meq_token_logprobs gives it, keeps the small
 * differences that a sum over an answer would round off. Rows in no answer get
 * a zero gradient. loss: device float; margins: device, pairs floats, the x_j.
 * pairs in 1..2^27, beta > 0, label_smoothing in 0..1. */
meq_status meq_preference_loss(const void* logits, int type, int64_t rows, int64_t cols, int64_t ld, const int64_t* targets,
                               const int64_t* starts, int64_t pairs, const float* ref_logp, const float* weights, float beta,
                               float label_smoothing, float* loss, float* margins, float* logp, void* grad, int64_t ld_grad,
                               const float* grad_scale, float* work, void* cuda_stream);

/* ---- norms ------------------------------------------------------------------
 * Layer norm and RMS norm of rows of activations (tokens), with the addition to
 * the residual stream, and their backward pass. Forward, for every row:
 *
 *   h = x + residual (rounded to its type; x itself without a residual)
 *   mu = mean_j h_j (RMS norm: 0),  rstd = 1 / sqrt(mean_j (h_j - mu)^2 + eps)
 *   y_j = (h_j - mu) rstd w_j + b_j
 *
 * and backward, with xhat = (h - mu) rstd and a = dy w:
 *
 *   dx = rstd (a - mean(a) - xhat mean(a xhat)) + dh      (RMS norm: no mean(a))
 *   dw = sum_rows dy xhat,  db = sum_rows dy
 *
 * dx is the gradient of h, which both x and the residual get; dh: what the
 * stream's later uses add to it.
 * x, residual, y, h, dy, dh, dx: device, rows x cols of meq_dtype `type`,
 *   consecutive columns, rows ld_* elements apart (>= cols); rows may start at
 *   any element. Fastest where all start at multiples of 16 bytes, next where
 *   the rows of all matrices lie in their 16 bytes alike (start and stride
 *   leave the same rest), as they do when allocated alike.
 * weight, bias: device, cols elements of weight_type (NULL: 1 and 0).
 * mean, rstd: device, rows floats. mean NULL selects RMS norm, in both calls.
 * In place: y may be x or the residual, h may be x or the residual (not what y
 *   is), dx may be dy, h or dh: the same pointer and row stride. Otherwise
 *   outputs must not overlap inputs or one another. y over x without a residual
 *   leaves no h for the backward pass.
 * Sums and statistics are fp32, in fixed orders: results repeat bit for bit. A
 * row whose sum of squares is not finite in fp32 gives NaN. rows may be 0.
 * Nothing is allocated, and the calls may come from several threads. Limits:
 * rows <= 2^27, cols <= 2^20, eps finite and > 0. */
meq_status meq_layer_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int type, int64_t rows, int64_t cols,
                          const void* weight, const void* bias, int weight_type, float eps, void* y, int64_t ld_y, void* h, int64_t ld_h,
                          float* mean, float* rstd, void* cuda_stream);
/* Floats of `work` for meq_layer_norm_grad. Host only. */
int64_t meq_layer_norm_work_floats(int64_t rows, int64_t cols);
/* dh: NULL, or added to dx. dweight, dbias: NULL, or device, cols elements of
 * grad_type, overwritten (zeros for no rows). work: device scratch of
 * meq_layer_norm_work_floats floats, 16-byte aligned, free again when the
 * enqueued kernels have run. Up to 65536 elements it may be NULL: a call that
 * needs it all the same (rows of the matrices that lie in their 16 bytes
 * differently, or too long for a block) is MEQ_ERR_INVALID_ARG, and nothing is
 * enqueued. */
meq_status meq_layer_norm_grad(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* dh, int64_t ld_dh, int type,
                               int64_t rows, int64_t cols, const void* weight, int weight_type, const float* mean, const float* rstd,
                               void* dx, int64_t ld_dx, void* dweight, void* dbias, int grad_type, float* work, void* cuda_stream);

/* ---- embedding ---------------------------------------------------------------
 * out_i = scale E[t_i] for n tokens t and a table E of vocab rows, and the
 * gradient of the table,
 *
 *   dE[v] = scale sum_{i: t_i = v} g_i,
 *
 * where g is the gradient of out. A negative token (padding) gives a row of
 * zeros and no gradient; one >= vocab a row of NaN and no gradient.
 * tokens: device, n int64. table, out, grad: device, of meq_dtype table_type,
 *   out_type and type, consecutive columns, rows ld_* elements apart (>= cols);
 *   rows may start at any element. Fastest where all start at multiples of 16
 *   bytes and cols is a multiple of 8. out must not overlap an input.
 * Sums are fp32, scaled and rounded once, in a fixed order (positions in turn,
 * in groups that depend on n and cols alone): results repeat bit for bit.
 * Nothing is allocated, and the calls may come from several threads. n may be 0.
 * Limits: n <= 2^27, vocab <= 2^28, cols <= 2^20. */
meq_status meq_embedding(const int64_t* tokens, int64_t n, const void* table, int table_type, int64_t vocab, int64_t cols, int64_t ld_table,
                         float scale, void* out, int out_type, int64_t ld_out, void* cuda_stream);
/* Floats of `work` for meq_embedding_grad. Host only. */
int64_t meq_embedding_work_floats(int64_t n, int64_t vocab, int64_t cols);
/* The gradient of the table into out (vocab rows of out_type): every row is
 * written, or with accumulate != 0 the sums are added to what the rows hold (a
 * table shared with the head, micro-batches) and the other rows left as they
 * are. work: device scratch of meq_embedding_work_floats floats, 16-byte
 * aligned, free again when the enqueued kernels have run. */
meq_status meq_embedding_grad(const void* grad, int type, int64_t n, int64_t cols, int64_t ld, const int64_t* tokens, int64_t vocab,
                              float scale, void* out, int out_type, int64_t ld_out, int accumulate, float* work, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* MEQ_H */

"""Thin ctypes binding of the C ABI (include/meq.h): MeqMuon, AdamW, the losses
of fine-tuning, norms and embedding.

Argument marshalling only: every step of the optimizers and every operator runs
in the CUDA library. There is no fallback: if libmeq.so is missing or fails to
load, importing this module raises.
"""
from __future__ import annotations

import array
import collections
import ctypes
import functools
import operator
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmeq.so")

MEQ_OK = 0
STATUS_NAMES = {
    0: "MEQ_OK", 1: "MEQ_ERR_INVALID_ARG", 2: "MEQ_ERR_OOM", 3: "MEQ_ERR_CUDA",
    4: "MEQ_ERR_NONFINITE", 5: "MEQ_ERR_TIMEOUT", 6: "MEQ_ERR_UNSUPPORTED", 7: "MEQ_ERR_CORRUPTED",
}
ROW, COL = 0, 1


class MeqShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class MeqOptions(ctypes.Structure):
    _fields_ = [
        ("rho", ctypes.c_float),
        ("ns_steps", ctypes.c_int),
        ("ns_a", ctypes.c_float),
        ("ns_b", ctypes.c_float),
        ("ns_c", ctypes.c_float),
        ("nesterov", ctypes.c_int),
        ("ns_fp16_mask", ctypes.c_uint32),
        ("tie_atol", ctypes.c_float),
        ("use_graph", ctypes.c_int),
        ("workspace_limit_bytes", ctypes.c_int64),
        ("wait_timeout_ms", ctypes.c_float),
        ("ns_cta_pair", ctypes.c_int),
        ("ns_x0_fused", ctypes.c_int),
        ("update_rule", ctypes.c_int),
        ("debug_canaries", ctypes.c_int),
        ("debug_skip_load", ctypes.c_int),
    ]


class MeqAdamWOptions(ctypes.Structure):
    _fields_ = [
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("state_bits", ctypes.c_int),
        ("param_type", ctypes.c_int),
        ("grad_type", ctypes.c_int),
    ]


EXPORTED = [
    "meq_default_options", "meq_state_bytes", "meq_init_state", "meq_step", "meq_sync", "meq_free",
    "meq_last_error", "meq_status_string", "meq_read_momentum", "meq_write_momentum",
    "meq_read_ns_output", "meq_read_stats", "meq_kernels_per_step", "meq_debug_wait_selftest",
    "meq_set_profiling", "meq_read_profile", "meq_row_col_stats_noalloc",
    "meq_init_state_kinds", "meq_state_bytes_kinds", "meq_ns_gemm_launches_per_step",
    "meq_read_direction_counts", "meq_reset_direction_counts", "meq_ns_cv_trajectory",
    "meq_check_canaries", "meq_canary_count", "meq_debug_corrupt_canary",
    "meq_step_prepare", "meq_step_apply", "meq_read_update", "meq_ns_flops_per_step",
    "meq_ns_gemm_tile_columns",
    "meq_adamw_default_options", "meq_adamw_state_bytes", "meq_adamw_init", "meq_adamw_grad_norm", "meq_adamw_step",
    "meq_adamw_state_ptrs", "meq_adamw_read_values", "meq_adamw_steps", "meq_adamw_set_steps", "meq_adamw_sync",
    "meq_adamw_free", "meq_adamw_last_error",
    "meq_token_logprobs", "meq_loss_work_floats", "meq_policy_loss", "meq_preference_loss",
    "meq_debug_loss_wait",
    "meq_layer_norm", "meq_layer_norm_work_floats", "meq_layer_norm_grad",
    "meq_embedding", "meq_embedding_work_floats", "meq_embedding_grad",
]
HIDDEN, REMAINING_2D, VECTOR = 0, 1, 2  # meq_kind
RULE_MEQMUON, RULE_MUON = 0, 1          # meq_update_rule
DTYPES = {"float32": 0, "bfloat16": 1, "float16": 2}  # meq_dtype


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2609_35701_gb300.build.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, F, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_double
    lib.meq_default_options.argtypes = [ctypes.POINTER(MeqOptions)]
    lib.meq_default_options.restype = None
    lib.meq_state_bytes.argtypes = [ctypes.POINTER(MeqShape), I, ctypes.POINTER(MeqOptions),
                                    ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
    lib.meq_state_bytes.restype = I
    lib.meq_init_state.argtypes = [ctypes.POINTER(MeqShape), I, ctypes.POINTER(MeqOptions), P, ctypes.POINTER(P)]
    lib.meq_init_state.restype = I
    lib.meq_step.argtypes = [ctypes.POINTER(P), ctypes.POINTER(P), P, ctypes.POINTER(MeqShape), I, F, F, F, F, P]
    lib.meq_step.restype = I
    lib.meq_step_prepare.argtypes = [ctypes.POINTER(P), P, ctypes.POINTER(MeqShape), I, F, F, F, F, P]
    lib.meq_step_prepare.restype = I
    lib.meq_step_apply.argtypes = [ctypes.POINTER(P), P, P]
    lib.meq_step_apply.restype = I
    lib.meq_sync.argtypes = [P]
    lib.meq_sync.restype = I
    lib.meq_free.argtypes = [P]
    lib.meq_free.restype = I
    lib.meq_last_error.argtypes = [P]
    lib.meq_last_error.restype = ctypes.c_char_p
    lib.meq_status_string.argtypes = [I]
    lib.meq_status_string.restype = ctypes.c_char_p
    lib.meq_read_momentum.argtypes = [P, I, P]
    lib.meq_read_momentum.restype = I
    lib.meq_write_momentum.argtypes = [P, I, P]
    lib.meq_write_momentum.restype = I
    lib.meq_read_ns_output.argtypes = [P, I, P]
    lib.meq_read_ns_output.restype = I
    lib.meq_read_update.argtypes = [P, I, P]
    lib.meq_read_update.restype = I
    lib.meq_read_stats.argtypes = [P, I, P, P, ctypes.POINTER(D), ctypes.POINTER(D), ctypes.POINTER(I)]
    lib.meq_read_stats.restype = I
    lib.meq_kernels_per_step.argtypes = [P]
    lib.meq_kernels_per_step.restype = I
    lib.meq_debug_wait_selftest.argtypes = [P, F]
    lib.meq_debug_wait_selftest.restype = I
    lib.meq_set_profiling.argtypes = [P, I]
    lib.meq_set_profiling.restype = I
    lib.meq_read_profile.argtypes = [P, P, ctypes.POINTER(ctypes.c_int64)]
    lib.meq_read_profile.restype = I
    lib.meq_row_col_stats_noalloc.argtypes = [P, ctypes.c_int64, ctypes.c_int64, F, F, P, P, P, P, P]
    lib.meq_row_col_stats_noalloc.restype = I
    lib.meq_init_state_kinds.argtypes = [ctypes.POINTER(MeqShape), P, I, ctypes.POINTER(MeqOptions), P,
                                         ctypes.POINTER(P)]
    lib.meq_init_state_kinds.restype = I
    lib.meq_state_bytes_kinds.argtypes = [ctypes.POINTER(MeqShape), P, I, ctypes.POINTER(MeqOptions),
                                          ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
    lib.meq_state_bytes_kinds.restype = I
    lib.meq_ns_gemm_launches_per_step.argtypes = [P]
    lib.meq_ns_gemm_launches_per_step.restype = I
    lib.meq_ns_gemm_tile_columns.argtypes = [P, I]
    lib.meq_ns_gemm_tile_columns.restype = I
    lib.meq_ns_flops_per_step.argtypes = [P]
    lib.meq_ns_flops_per_step.restype = D
    lib.meq_read_direction_counts.argtypes = [P, I, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    lib.meq_read_direction_counts.restype = I
    lib.meq_reset_direction_counts.argtypes = [P]
    lib.meq_reset_direction_counts.restype = I
    lib.meq_ns_cv_trajectory.argtypes = [P, ctypes.c_int64, ctypes.c_int64, I, F, ctypes.POINTER(MeqOptions),
                                         ctypes.POINTER(D), ctypes.POINTER(D), P]
    lib.meq_ns_cv_trajectory.restype = I
    lib.meq_check_canaries.argtypes = [P, ctypes.POINTER(ctypes.c_int64)]
    lib.meq_check_canaries.restype = I
    lib.meq_canary_count.argtypes = [P]
    lib.meq_canary_count.restype = I
    lib.meq_debug_corrupt_canary.argtypes = [P, I]
    lib.meq_debug_corrupt_canary.restype = I
    S, PP, I64 = ctypes.c_size_t, ctypes.POINTER(P), ctypes.c_int64
    lib.meq_adamw_default_options.argtypes = [ctypes.POINTER(MeqAdamWOptions)]
    lib.meq_adamw_default_options.restype = None
    lib.meq_adamw_state_bytes.argtypes = [ctypes.POINTER(MeqShape), I, ctypes.POINTER(MeqAdamWOptions), ctypes.POINTER(S),
                                          ctypes.POINTER(S)]
    lib.meq_adamw_state_bytes.restype = I
    lib.meq_adamw_init.argtypes = [ctypes.POINTER(MeqShape), P, I, ctypes.POINTER(MeqAdamWOptions), P, PP]
    lib.meq_adamw_init.restype = I
    lib.meq_adamw_grad_norm.argtypes = [P, P, F, P, P]
    lib.meq_adamw_grad_norm.restype = I
    lib.meq_adamw_step.argtypes = [P, P, P, P, F, F, P, P]
    lib.meq_adamw_step.restype = I
    lib.meq_adamw_state_ptrs.argtypes = [P, PP, PP, PP, PP, ctypes.POINTER(I64)]
    lib.meq_adamw_state_ptrs.restype = I
    lib.meq_adamw_read_values.argtypes = [P, P, P, P]
    lib.meq_adamw_read_values.restype = I
    lib.meq_adamw_steps.argtypes = [P, ctypes.POINTER(I64)]
    lib.meq_adamw_steps.restype = I
    lib.meq_adamw_set_steps.argtypes = [P, I64]
    lib.meq_adamw_set_steps.restype = I
    lib.meq_adamw_sync.argtypes = [P]
    lib.meq_adamw_sync.restype = I
    lib.meq_adamw_free.argtypes = [P]
    lib.meq_adamw_free.restype = I
    lib.meq_adamw_last_error.argtypes = [P]
    lib.meq_adamw_last_error.restype = ctypes.c_char_p
    lib.meq_token_logprobs.argtypes = [P, I, I64, I64, I64, P, P, P, P]
    lib.meq_token_logprobs.restype = I
    lib.meq_loss_work_floats.argtypes = [I64, I64]
    lib.meq_loss_work_floats.restype = I64
    lib.meq_policy_loss.argtypes = [P, I, I64, I64, I64, P, P, P, P, P, F, F, F, P, P, P, I64, P, P, P]
    lib.meq_policy_loss.restype = I
    lib.meq_preference_loss.argtypes = [P, I, I64, I64, I64, P, P, I64, P, P, F, F, P, P, P, P, I64, P, P, P]
    lib.meq_preference_loss.restype = I
    lib.meq_debug_loss_wait.argtypes = [F, I64]
    lib.meq_debug_loss_wait.restype = I
    lib.meq_layer_norm.argtypes = [P, I64, P, I64, I, I64, I64, P, P, I, F, P, I64, P, I64, P, P, P]
    lib.meq_layer_norm.restype = I
    lib.meq_layer_norm_work_floats.argtypes = [I64, I64]
    lib.meq_layer_norm_work_floats.restype = I64
    lib.meq_layer_norm_grad.argtypes = [P, I64, P, I64, P, I64, I, I64, I64, P, I, P, P, P, I64, P, P, I, P, P]
    lib.meq_layer_norm_grad.restype = I
    lib.meq_embedding.argtypes = [P, I64, P, I, I64, I64, I64, F, P, I, I64, P]
    lib.meq_embedding.restype = I
    lib.meq_embedding_work_floats.argtypes = [I64, I64, I64]
    lib.meq_embedding_work_floats.restype = I64
    lib.meq_embedding_grad.argtypes = [P, I, I64, I64, I64, P, I64, F, P, I, I64, I, P, P]
    lib.meq_embedding_grad.restype = I
    return lib


lib = _load()


class MeqError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def default_options(**overrides):
    o = MeqOptions()
    lib.meq_default_options(ctypes.byref(o))
    for k, v in overrides.items():
        if not hasattr(o, k):
            raise KeyError(k)
        setattr(o, k, v)
    return o


def _shape_array(shapes):
    arr = (MeqShape * len(shapes))()
    for i, (r, c) in enumerate(shapes):
        arr[i].rows, arr[i].cols = int(r), int(c)
    return arr


def _kind_array(kinds, n):
    if kinds is None:
        return None
    if len(kinds) != n:
        raise ValueError("one kind per shape")
    return (ctypes.c_int * n)(*[int(k) for k in kinds])


def state_bytes(shapes, kinds=None, **opts):
    """(persistent, workspace) bytes for a shape list, computed on the host."""
    p, w = ctypes.c_size_t(), ctypes.c_size_t()
    o = default_options(**opts)
    st = lib.meq_state_bytes_kinds(_shape_array(shapes), _kind_array(kinds, len(shapes)), len(shapes), ctypes.byref(o),
                                   ctypes.byref(p), ctypes.byref(w))
    if st != MEQ_OK:
        raise MeqError(st, lib.meq_last_error(None).decode())
    return p.value, w.value


def ns_cv_trajectory(H, steps=20, eps=1e-7, stream=None, **opts):
    """(gamma_r, gamma_c) of the NS iterates X_0..X_steps of a CUDA fp32
    matrix H (meq_ns_cv_trajectory)."""
    if H.dim() != 2:
        raise ValueError("H must be a matrix")
    _require_cuda(H, "float32", H.shape[0] * H.shape[1], "H")
    gr = (ctypes.c_double * (steps + 1))()
    gc = (ctypes.c_double * (steps + 1))()
    o = default_options(**opts)
    st = lib.meq_ns_cv_trajectory(H.data_ptr(), H.shape[0], H.shape[1], int(steps), float(eps), ctypes.byref(o),
                                  gr, gc, _stream_handle(stream))
    if st != MEQ_OK:
        raise MeqError(st, lib.meq_last_error(None).decode())
    return np.array(list(gr)), np.array(list(gc))


def row_col_stats_noalloc(U, r, c, gammas, direction, eps=1e-7, tie_atol=1e-6, stream=None):
    """Statistics of one CUDA fp32 matrix U into caller-provided CUDA tensors
    r (rows), c (cols), gammas (2 x float64) and direction (1 x int32),
    without any device allocation (see include/meq.h). Returns the status."""
    rows, cols = U.shape
    _require_cuda(U, "float32", rows * cols, "U")
    _require_cuda(r, "float32", rows, "r", U.device.index)
    _require_cuda(c, "float32", cols, "c", U.device.index)
    _require_cuda(gammas, "float64", 2, "gammas", U.device.index)
    _require_cuda(direction, "int32", 1, "direction", U.device.index)
    return lib.meq_row_col_stats_noalloc(ctypes.c_void_p(U.data_ptr()), rows, cols, float(eps), float(tie_atol),
                                         ctypes.c_void_p(r.data_ptr()), ctypes.c_void_p(c.data_ptr()),
                                         ctypes.c_void_p(gammas.data_ptr()), ctypes.c_void_p(direction.data_ptr()),
                                         _stream_handle(stream))


def _require_cuda(t, dtype_name, numel, what, device=None):
    """Raises unless t is a contiguous CUDA tensor of the given dtype (a
    torch dtype name) and element count (on `device` when given): the library
    only sees a pointer, so a tensor of the wrong size or type would be read
    or written past its end."""
    if not t.is_cuda or str(t.dtype) != "torch." + dtype_name or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype_name} CUDA tensor")
    if t.numel() != numel:
        raise ValueError(f"{what} has {t.numel()} elements, expected {numel}")
    if device is not None and t.device.index != device:
        raise ValueError(f"{what} is on cuda:{t.device.index}, the state on cuda:{device}")


def _stream_handle(stream, device=None):
    """The stream's handle, or that of the current stream (of `device`, if the caller knows the current one)."""
    if stream is None:
        import torch
        # the raw handle: torch.cuda.current_stream() builds a Stream object, which takes longer than a launch
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device))
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _empty(size, dtype, device, stream):
    """An uninitialised CUDA tensor whose memory belongs to the stream that the call runs on."""
    import torch

    if stream is None:
        return torch.empty(size, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(size, dtype=dtype, device=device)


class MeqMuon:
    """MeqMuon state for a fixed list of parameters (rows, cols); kinds (one
    meq_kind per entry, default all HIDDEN) select the branch of Algorithm 1."""

    def __init__(self, shapes, stream=None, kinds=None, **opts):
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.kinds = [HIDDEN] * len(self.shapes) if kinds is None else [int(k) for k in kinds]
        self._shape_arr = _shape_array(self.shapes)
        self._opts = default_options(**opts)
        import torch

        self._device = torch.cuda.current_device()  # the state lives on the current device
        self._st = ctypes.c_void_p()
        s = lib.meq_init_state_kinds(self._shape_arr, _kind_array(self.kinds, len(self.shapes)), len(self.shapes),
                                     ctypes.byref(self._opts), _stream_handle(stream), ctypes.byref(self._st))
        if s != MEQ_OK:
            raise MeqError(s, lib.meq_last_error(None).decode())
        n = len(self.shapes)
        self._pp = (ctypes.c_void_p * n)()
        self._gp = (ctypes.c_void_p * n)()

    def _check(self, s):
        if s != MEQ_OK:
            raise MeqError(s, lib.meq_last_error(self._st).decode())

    @property
    def kernels_per_step(self):
        return lib.meq_kernels_per_step(self._st)

    @property
    def ns_gemm_launches_per_step(self):
        return lib.meq_ns_gemm_launches_per_step(self._st)

    @property
    def ns_gemm_tile_columns(self):
        """Tile width of each Newton-Schulz launch (meq_ns_gemm_tile_columns)."""
        return [lib.meq_ns_gemm_tile_columns(self._st, i) for i in range(self.ns_gemm_launches_per_step)]

    @property
    def ns_flops_per_step(self):
        return lib.meq_ns_flops_per_step(self._st)

    def step_ptrs(self, param_ptrs, grad_ptrs, lr, momentum, weight_decay, eps=1e-7, stream=None):
        """One step given raw device pointers (ints)."""
        for i, (p, g) in enumerate(zip(param_ptrs, grad_ptrs)):
            self._pp[i] = p
            self._gp[i] = g
        self._check(lib.meq_step(self._pp, self._gp, self._st, self._shape_arr, len(self.shapes), float(lr),
                                 float(momentum), float(weight_decay), float(eps), _stream_handle(stream)))

    def step(self, params, grads, lr, momentum, weight_decay, eps=1e-7, stream=None):
        """One step on lists of contiguous fp32 CUDA tensors (params updated in place)."""
        if len(params) != len(self.shapes) or len(grads) != len(self.shapes):
            raise ValueError("params / grads must have one tensor per matrix")
        self._check_tensors(params, "params")
        self._check_tensors(grads, "grads")
        self.step_ptrs([p.data_ptr() for p in params], [g.data_ptr() for g in grads], lr, momentum, weight_decay,
                       eps, stream)

    def _check_tensors(self, ts, what):
        for i, (t, (r, c)) in enumerate(zip(ts, self.shapes)):
            _require_cuda(t, "float32", r * c, f"{what}[{i}]", self._device)

    def step_prepare(self, grads, lr, momentum, weight_decay, eps=1e-7, stream=None):
        """First half of a step (meq_step_prepare): momentum, Newton-Schulz and
        statistics for these gradients; the parameters are not touched."""
        if len(grads) != len(self.shapes):
            raise ValueError("grads must have one tensor per matrix")
        self._check_tensors(grads, "grads")
        n = len(self.shapes)
        for i, g in enumerate(grads):
            self._gp[i] = g.data_ptr()
        self._check(lib.meq_step_prepare(self._gp, self._st, self._shape_arr, n, float(lr), float(momentum),
                                         float(weight_decay), float(eps), _stream_handle(stream)))

    def step_apply(self, params, stream=None):
        """Second half of a step (meq_step_apply): the update of params."""
        if len(params) != len(self.shapes):
            raise ValueError("params must have one tensor per matrix")
        self._check_tensors(params, "params")
        for i, p in enumerate(params):
            self._pp[i] = p.data_ptr()
        self._check(lib.meq_step_apply(self._pp, self._st, _stream_handle(stream)))

    def sync(self):
        self._check(lib.meq_sync(self._st))

    def read_momentum(self, i):
        r, c = self.shapes[i]
        out = np.empty((r, c), np.float32)
        self._check(lib.meq_read_momentum(self._st, i, out.ctypes.data))
        return out

    def write_momentum(self, i, arr):
        r, c = self.shapes[i]
        a = np.ascontiguousarray(arr, dtype=np.float32)
        if a.shape != (r, c):
            raise ValueError(f"momentum {i} must have shape {(r, c)}, got {a.shape}")
        self._check(lib.meq_write_momentum(self._st, i, a.ctypes.data))

    def read_ns_output(self, i):
        r, c = self.shapes[i]
        out = np.empty((r, c), np.float32)
        self._check(lib.meq_read_ns_output(self._st, i, out.ctypes.data))
        return out

    def read_update(self, i):
        """The normalised update U~ the last step applied to entry i (meq_read_update)."""
        r, c = self.shapes[i]
        out = np.empty((r, c), np.float32)
        self._check(lib.meq_read_update(self._st, i, out.ctypes.data))
        return out

    def read_stats(self, i):
        r, c = self.shapes[i]
        rv = np.empty(r, np.float32)
        cv = np.empty(c, np.float32)
        gr, gc, d = ctypes.c_double(), ctypes.c_double(), ctypes.c_int()
        self._check(lib.meq_read_stats(self._st, i, rv.ctypes.data, cv.ctypes.data, ctypes.byref(gr),
                                       ctypes.byref(gc), ctypes.byref(d)))
        return {"r": rv, "c": cv, "gamma_r": gr.value, "gamma_c": gc.value, "direction": d.value}

    def read_direction_counts(self, i):
        """(row choices, column choices) of Eq. (11) for hidden weight i."""
        r, c = ctypes.c_int64(), ctypes.c_int64()
        self._check(lib.meq_read_direction_counts(self._st, i, ctypes.byref(r), ctypes.byref(c)))
        return r.value, c.value

    def check_canaries(self):
        """Raises MeqError (MEQ_ERR_CORRUPTED) if a workspace guard band changed."""
        off = ctypes.c_int64()
        self._check(lib.meq_check_canaries(self._st, ctypes.byref(off)))

    @property
    def canary_count(self):
        return lib.meq_canary_count(self._st)

    def reset_direction_counts(self):
        self._check(lib.meq_reset_direction_counts(self._st))

    def set_profiling(self, enable):
        self._check(lib.meq_set_profiling(self._st, int(bool(enable))))

    PHASES = ("momentum", "cast_x0", "ns_gemm", "stats", "apply")

    def read_profile(self):
        """Summed per-phase milliseconds and the number of profiled steps."""
        ms = (ctypes.c_double * 5)()
        n = ctypes.c_int64()
        self._check(lib.meq_read_profile(self._st, ms, ctypes.byref(n)))
        return dict(zip(self.PHASES, list(ms))), n.value

    def wait_selftest(self, timeout_ms=200.0):
        """Returns the status of the bounded-wait self test (expected MEQ_ERR_TIMEOUT)."""
        return lib.meq_debug_wait_selftest(self._st, float(timeout_ms))

    def close(self):
        if self._st:
            lib.meq_free(self._st)
            self._st = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------- AdamW
def _adamw_options(o, param_dtype, grad_dtype):
    for what, name in (("param_dtype", param_dtype), ("grad_dtype", grad_dtype)):
        if name not in DTYPES:
            raise ValueError(f"{what} must be one of {sorted(DTYPES)}")
    opts = MeqAdamWOptions()
    lib.meq_adamw_default_options(ctypes.byref(opts))
    for k, v in o.items():
        if not hasattr(opts, k):
            raise KeyError(k)
        setattr(opts, k, v)
    opts.param_type, opts.grad_type = DTYPES[param_dtype], DTYPES[grad_dtype]
    return opts


def adamw_state_bytes(shapes, param_dtype="float32", grad_dtype="float32", **opts):
    """(persistent, workspace) bytes of an AdamW state, computed on the host (meq_adamw_state_bytes)."""
    p, w = ctypes.c_size_t(), ctypes.c_size_t()
    o = _adamw_options(opts, param_dtype, grad_dtype)
    s = lib.meq_adamw_state_bytes(_shape_array(shapes), len(shapes), ctypes.byref(o), ctypes.byref(p), ctypes.byref(w))
    if s != MEQ_OK:
        raise MeqError(s, lib.meq_adamw_last_error(None).decode())
    return p.value, w.value


_dtype_of = operator.attrgetter("dtype")


class _DeviceArray:
    """Device memory of a state as torch.as_tensor takes it; keeps its owner alive."""

    def __init__(self, owner, ptr, shape, typestr):
        self._owner = owner
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": shape, "typestr": typestr, "version": 2}


class AdamW:
    """AdamW over a fixed list of parameters (rows, cols), with moments in 32
    or 8 bits (meq_adamw_init). decay: a factor of the weight decay per entry
    (default 1); options beta1, beta2, eps, state_bits. steps, set_steps, sync
    and close wait for the stream of the last call, or, once a call has been
    captured into a graph, for the device."""

    BLOCK = 256  # each entry's moments start at a multiple of this many elements

    def __init__(self, shapes, stream=None, decay=None, param_dtype="float32", grad_dtype="float32", **opts):
        import torch

        self.shapes = [(int(r), int(c)) for r, c in shapes]
        n = len(self.shapes)
        if decay is not None and len(decay) != n:
            raise ValueError("one decay factor per shape")
        self._opts = _adamw_options(opts, param_dtype, grad_dtype)
        self._param_dtype, self._grad_dtype = getattr(torch, param_dtype), getattr(torch, grad_dtype)
        self._numels = [r * c for r, c in self.shapes]
        self._device = torch.cuda.current_device()
        self._st = ctypes.c_void_p()
        d = None if decay is None else (ctypes.c_float * n)(*[float(x) for x in decay])
        s = lib.meq_adamw_init(_shape_array(self.shapes), d, n, ctypes.byref(self._opts), _stream_handle(stream),
                               ctypes.byref(self._st))
        if s != MEQ_OK:
            raise MeqError(s, lib.meq_adamw_last_error(None).decode())
        self.offsets, at = [], 0  # first element of each entry in the state's arrays
        for k in self._numels:
            self.offsets.append(at)
            at += -(-k // self.BLOCK) * self.BLOCK
        self._cuda = torch.device("cuda", self._device)
        p, size = [ctypes.c_void_p() for _ in range(4)], ctypes.c_int64()
        self._check(lib.meq_adamw_state_ptrs(self._st, *[ctypes.byref(x) for x in p], ctypes.byref(size)))
        p, k = [x.value for x in p], size.value
        if self._opts.state_bits == 32:
            self._arrays = [("m", p[0], k, "<f4"), ("v", p[1], k, "<f4")]
        else:
            self._arrays = [("m_code", p[0], k, "|i1"), ("r_code", p[1], k, "|u1"), ("m_scale", p[2], k // self.BLOCK, "<f4"),
                            ("r_scale", p[3], k // self.BLOCK, "<f4")]

    def _check(self, s):
        if s != MEQ_OK:
            raise MeqError(s, lib.meq_adamw_last_error(self._st).decode())

    def _pointers(self, ts, dtype, what):
        """An array of the tensors' pointers. The checks go over the list a property at a time, which
        takes a third of the time that a loop over the tensors does."""
        import torch

        T, n = torch.Tensor, len(ts)
        if n != len(self._numels):
            raise ValueError(f"{what} must have one tensor per entry")
        if not (list(map(T.numel, ts)) == self._numels and all(map(T.is_contiguous, ts)) and
                set(map(_dtype_of, ts)) == {dtype} and set(map(T.get_device, ts)) == {self._device}):
            for i, (t, k) in enumerate(zip(ts, self._numels)):
                _require_cuda(t, str(dtype)[6:], k, f"{what}[{i}]", self._device)
        return array.array("Q", map(T.data_ptr, ts))

    def grad_norm(self, grads, max_norm=float("inf"), out=None, stream=None):
        """(norm, clipping coefficient) of the gradients as a CUDA tensor of two floats, without a host sync."""
        if out is None:
            import torch

            out = _empty(2, torch.float32, self._device, stream)
        else:
            _require_cuda(out, "float32", 2, "out", self._device)
        g = self._pointers(grads, self._grad_dtype, "grads")
        self._check(lib.meq_adamw_grad_norm(g.buffer_info()[0], self._st, float(max_norm), out.data_ptr(),
                                            _stream_handle(stream)))
        return out

    def step(self, params, grads, lr, weight_decay=0.0, grad_scale=None, copies=None, stream=None):
        """One step on lists of contiguous CUDA tensors (params updated in place).
        grad_scale: a CUDA float32 tensor of one element that multiplies the
        gradients (not finite: the step is skipped); copies: bf16 tensors that
        receive the updated parameters. A backward pass still to come that has
        saved a parameter or copy raises."""
        if grad_scale is not None:
            _require_cuda(grad_scale, "float32", 1, "grad_scale", self._device)
        import torch

        p = self._pointers(params, self._param_dtype, "params")
        g = self._pointers(grads, self._grad_dtype, "grads")
        c = None
        if copies is not None:
            c = self._pointers(copies, torch.bfloat16, "copies")
        self._check(lib.meq_adamw_step(p.buffer_info()[0], g.buffer_info()[0], None if c is None else c.buffer_info()[0],
                                       self._st, float(lr), float(weight_decay),
                                       None if grad_scale is None else grad_scale.data_ptr(), _stream_handle(stream)))
        written = torch.autograd.graph.increment_version  # through pointers, which autograd does not see
        written(params)
        if copies is not None:
            written(copies)

    def state(self):
        """The state's own arrays as CUDA tensors: m and v, or m_code, r_code and
        their scales per 256 elements (meq_adamw_state_ptrs); copy them to
        checkpoint and copy into them to resume."""
        import torch

        if not self._st:
            raise MeqError(1, "the state is closed")
        return {name: torch.as_tensor(_DeviceArray(self, ptr, (size,), ts), device=self._cuda) for name, ptr, size, ts in self._arrays}

    def read_values(self, m=None, v=None, stream=None):
        """(m, v) as fp32 CUDA tensors laid out as the state's arrays (entry i at offsets[i])."""
        import torch

        k = self.offsets[-1] + -(-self._numels[-1] // self.BLOCK) * self.BLOCK
        m = _empty(k, torch.float32, self._device, stream) if m is None else m
        v = _empty(k, torch.float32, self._device, stream) if v is None else v
        _require_cuda(m, "float32", k, "m", self._device)
        _require_cuda(v, "float32", k, "v", self._device)
        self._check(lib.meq_adamw_read_values(self._st, ctypes.c_void_p(m.data_ptr()), ctypes.c_void_p(v.data_ptr()),
                                              _stream_handle(stream)))
        return m, v

    @property
    def steps(self):
        """Steps done, skipped ones not counted (waits for them)."""
        n = ctypes.c_int64()
        self._check(lib.meq_adamw_steps(self._st, ctypes.byref(n)))
        return n.value

    def set_steps(self, steps):
        self._check(lib.meq_adamw_set_steps(self._st, int(steps)))

    def sync(self):
        self._check(lib.meq_adamw_sync(self._st))

    def close(self):
        if self._st:
            lib.meq_adamw_free(self._st)
            self._st = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# --------------------------------------------------------------------- losses
TokenLogprobs = collections.namedtuple("TokenLogprobs", "logp lse")
PreferenceLoss = collections.namedtuple("PreferenceLoss", "loss margins logp grad")


class PolicyLoss(collections.namedtuple("PolicyLoss", "sums logp grad")):
    """sums: the loss, its surrogate and KL parts, the clipped weight."""

    __slots__ = ()

    @property
    def loss(self):
        return self.sums[0]


def _logits_args(logits, what="logits"):
    """(meq_dtype, rows, cols, row stride) of a CUDA matrix whose columns are consecutive."""
    kind = DTYPES.get(str(logits.dtype)[6:])
    if kind is None or not logits.is_cuda or logits.dim() != 2:
        raise ValueError(f"{what} must be a CUDA matrix of one of {sorted(DTYPES)}")
    rows, cols = logits.shape
    ld, step = logits.stride()
    if cols < 1 or (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{what} must have consecutive columns in rows that do not overlap")
    return kind, rows, cols, max(ld, cols)


def _vector(t, dtype, n, device, what):
    """The device pointer of a contiguous CUDA vector, or None."""
    if t is None:
        return None
    if not (t.dtype is dtype and t.get_device() == device and t.numel() == n and t.is_contiguous()):
        _require_cuda(t, str(dtype)[6:], n, what, device)
    return t.data_ptr()


def _grad_for(logits, rows, cols, ld, grad, stream):
    """The gradient's tensor, its pointer and row stride: none, the given one, or
    (True) a new one whose rows lie in their 16 bytes as the logits' do."""
    if grad is None or grad is False:
        return None, None, 0
    if grad is True:
        n = 16 // logits.element_size()
        lead, ldg = logits.data_ptr() % 16 // logits.element_size(), cols + (ld - cols) % n
        grad = _empty(rows * ldg + n, logits.dtype, logits.device, stream).as_strided((rows, cols), (ldg, 1), lead)
        return grad, grad.data_ptr(), ldg
    if grad.shape != logits.shape or grad.dtype is not logits.dtype or grad.device != logits.device:
        raise ValueError("grad must have the logits' shape, type and device")
    return grad, grad.data_ptr(), _logits_args(grad, "grad")[3]


def _current_device(t, what):
    import torch

    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError(f"{what} is on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    return device


def _check_call(s):
    if s != MEQ_OK:
        raise MeqError(s, lib.meq_last_error(None).decode())


def debug_loss_wait(timeout_ms=0.0, withheld_row=-1):
    """Diagnostic (meq_debug_loss_wait): the limit of the loss kernels' waits and a row whose data never comes."""
    _check_call(lib.meq_debug_loss_wait(float(timeout_ms), int(withheld_row)))


def token_logprobs(logits, targets, stream=None):
    """Log-probabilities of the target tokens and the rows' log-sum-exp
    (meq_token_logprobs). logits: CUDA matrix, fp32, bf16 or fp16, one row per
    token; targets: int64, negative where a row is not scored."""
    import torch

    kind, rows, cols, ld = _logits_args(logits)
    device = _current_device(logits, "logits")
    t = _vector(targets, torch.int64, rows, device, "targets")
    logp, lse = _empty(rows, torch.float32, logits.device, stream), _empty(rows, torch.float32, logits.device, stream)
    _check_call(lib.meq_token_logprobs(logits.data_ptr(), kind, rows, cols, ld, t, logp.data_ptr(), lse.data_ptr(),
                                       _stream_handle(stream, device)))
    return TokenLogprobs(logp, lse)


def policy_loss(logits, targets, old_logp, advantages, weights=None, ref_logp=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                grad=None, grad_scale=None, stream=None):
    """The clipped policy loss with a KL term and, if asked for, the gradient of
    the logits (meq_policy_loss). grad: True for a new tensor, or the tensor to
    write (it may be logits, unless autograd has saved them for a backward pass
    to come, which then raises). sums holds the loss, its surrogate and KL parts
    and the clipped weight; loss is the first of them."""
    import torch

    f32 = torch.float32
    kind, rows, cols, ld = _logits_args(logits)
    device, where = _current_device(logits, "logits"), logits.device
    old, adv = _vector(old_logp, f32, rows, device, "old_logp"), _vector(advantages, f32, rows, device, "advantages")
    w, ref = _vector(weights, f32, rows, device, "weights"), _vector(ref_logp, f32, rows, device, "ref_logp")
    t = _vector(targets, torch.int64, rows, device, "targets")
    scale = _vector(grad_scale, f32, 1, device, "grad_scale")
    given, (grad, g, ldg) = grad, _grad_for(logits, rows, cols, ld, grad, stream)
    work = _empty(lib.meq_loss_work_floats(rows, 0), f32, where, stream)
    sums, logp = _empty(4, f32, where, stream), _empty(rows, f32, where, stream)
    _check_call(lib.meq_policy_loss(logits.data_ptr(), kind, rows, cols, ld, t, old, adv, w, ref, float(clip_low),
                                    float(clip_high), float(kl_coef), sums.data_ptr(), logp.data_ptr(), g, ldg, scale,
                                    work.data_ptr(), _stream_handle(stream, device)))
    if grad is not None and grad is given:
        torch.autograd.graph.increment_version(grad)  # written through its pointer, which autograd does not see
    return PolicyLoss(sums, logp, grad)


def preference_loss(logits, targets, starts, ref_logp, weights=None, beta=0.1, label_smoothing=0.0, grad=None, grad_scale=None,
                    stream=None):
    """The paired preference loss and, if asked for, the gradient of the logits
    (meq_preference_loss). starts: int64 CUDA vector of 2 pairs + 1 row offsets,
    preferred and other answer in turn; grad as in policy_loss."""
    import torch

    f32 = torch.float32
    kind, rows, cols, ld = _logits_args(logits)
    device, where = _current_device(logits, "logits"), logits.device
    pairs = starts.numel() // 2
    if pairs < 1 or starts.numel() != 2 * pairs + 1:
        raise ValueError("starts must hold 2 pairs + 1 offsets")
    st = _vector(starts, torch.int64, 2 * pairs + 1, device, "starts")
    ref, w = _vector(ref_logp, f32, rows, device, "ref_logp"), _vector(weights, f32, rows, device, "weights")
    t = _vector(targets, torch.int64, rows, device, "targets")
    scale = _vector(grad_scale, f32, 1, device, "grad_scale")
    given, (grad, g, ldg) = grad, _grad_for(logits, rows, cols, ld, grad, stream)
    work = _empty(lib.meq_loss_work_floats(rows, pairs), f32, where, stream)
    logp, margins, loss = _empty(rows, f32, where, stream), _empty(pairs, f32, where, stream), _empty((), f32, where, stream)
    _check_call(lib.meq_preference_loss(logits.data_ptr(), kind, rows, cols, ld, t, st, pairs, ref, w, float(beta),
                                        float(label_smoothing), loss.data_ptr(), margins.data_ptr(), logp.data_ptr(), g, ldg,
                                        scale, work.data_ptr(), _stream_handle(stream, device)))
    if grad is not None and grad is given:
        torch.autograd.graph.increment_version(grad)  # written through its pointer, which autograd does not see
    return PreferenceLoss(loss, margins, logp, grad)


# ---------------------------------------------------------- norms and embedding
LayerNorm = collections.namedtuple("LayerNorm", "y h mean rstd")
RmsNorm = collections.namedtuple("RmsNorm", "y h rstd")
LayerNormGrad = collections.namedtuple("LayerNormGrad", "dx dweight dbias")
RmsNormGrad = collections.namedtuple("RmsNormGrad", "dx dweight")


def _matrix(t, dtype, shape, device, what):
    """Pointer and row stride of a CUDA matrix of the given dtype, shape and device (None: no matrix)."""
    if t is None:
        return None, 0
    if t.dtype is dtype and t.shape == shape and t.get_device() == device:
        ld, step = t.stride()
        if step == 1 and ld >= shape[1]:  # the usual case: six properties, each 0.1 us and more to ask
            return t.data_ptr(), ld
        return t.data_ptr(), _logits_args(t, what)[3]
    raise ValueError(f"{what} must be a {tuple(shape)} CUDA matrix of {dtype} on cuda:{device}")


_KINDS = {}  # meq_dtype by torch dtype, filled as they come: torch is not imported before it is used


def _kind(t, what):
    kind = _KINDS.get(t.dtype)
    if kind is None:
        kind = DTYPES.get(str(t.dtype)[6:])
        if kind is None:
            raise ValueError(f"{what} must be of one of {sorted(DTYPES)}")
        _KINDS[t.dtype] = kind
    return kind


def _columns(t, cols, device, what, dtype=None):
    """Pointer and meq_dtype of a contiguous CUDA vector of cols elements (None: no vector)."""
    if t is None:
        return None, 0
    kind = _kind(t, what)
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{what} must be of {dtype}")
    if not (t.numel() == cols and t.get_device() == device and t.is_contiguous()):
        _require_cuda(t, str(t.dtype)[6:], cols, what, device)
    return t.data_ptr(), kind


# What the calls below use of torch, bound by the first of them: an import in every call takes longer than the lookups.
_f32 = _i64 = _new = _raw_stream = _device_now = _increment = None


def _bind_torch():
    global _f32, _i64, _new, _raw_stream, _device_now, _increment
    import torch

    _i64, _new, _raw_stream, _device_now = torch.int64, torch.empty, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    _increment = torch.autograd.graph.increment_version  # of tensors that a call has written through their pointers
    _f32 = torch.float32


def _first(t, what):
    """(meq_dtype, shape, row stride, device) of a call's first matrix, which has to be on the current device."""
    if _f32 is None:
        _bind_torch()
    kind, shape, device = _KINDS.get(t.dtype), t.shape, t.get_device()
    if kind is None:
        kind = _kind(t, what)
    if device < 0 or len(shape) != 2:
        _logits_args(t, what)
    if device != _device_now():
        _current_device(t, what)
    ld, step = t.stride()
    if step != 1 or ld < shape[1]:
        ld = _logits_args(t, what)[3]
    return kind, shape, ld, device


def _memory(size, dtype, device, stream):
    return _new(size, dtype=dtype, device=device) if stream is None else _empty(size, dtype, device, stream)


def _stream(stream, device):
    return _raw_stream(device) if stream is None else _stream_handle(stream)


_FEW_ELEMENTS = 65536  # up to which meq_layer_norm_grad may do without work


@functools.lru_cache(maxsize=256)
def _norm_work(rows, cols):
    return lib.meq_layer_norm_work_floats(rows, cols)


def _norm(x, weight, bias, residual, eps, y, h, stream, centred):
    kind, shape, ld, device = _first(x, "x")
    rows, cols = shape
    dtype, where, f32 = x.dtype, x.device, _f32
    r, ld_r = _matrix(residual, dtype, shape, device, "residual")
    w, weight_kind = _columns(weight, cols, device, "weight")
    if bias is None:
        b = None
    else:
        b, weight_kind = _columns(bias, cols, device, "bias", None if weight is None else weight.dtype)
    given = [t for t in (y, h) if t is not None]
    if y is None:
        y, ld_y = _memory(shape, dtype, where, stream), cols
        yp = y.data_ptr()
    else:
        yp, ld_y = _matrix(y, dtype, shape, device, "y")
    if residual is None:
        if h is not None:
            raise ValueError("h is written with a residual only")
        # y over x leaves nothing that the backward pass could read
        h, hp, ld_h = None if yp == x.data_ptr() and rows else x, None, 0
    elif h is None:
        h, ld_h = _memory(shape, dtype, where, stream), cols
        hp = h.data_ptr()
    else:
        hp, ld_h = _matrix(h, dtype, shape, device, "h")
    mean = mp = None
    if centred:
        mean = _memory(rows, f32, where, stream)
        mp = mean.data_ptr()
    rstd = _memory(rows, f32, where, stream)
    _check_call(lib.meq_layer_norm(x.data_ptr(), ld, r, ld_r, kind, rows, cols, w, b, weight_kind, float(eps), yp, ld_y, hp, ld_h, mp,
                                   rstd.data_ptr(), _stream(stream, device)))
    if given:
        _increment(given)
    return y, h, mean, rstd


def layer_norm(x, weight=None, bias=None, residual=None, eps=1e-5, y=None, h=None, stream=None):
    """Layer norm of the rows of x, or of h = x + residual (meq_layer_norm). x:
    CUDA matrix, fp32, bf16 or fp16, one row per token; weight, bias: vectors of
    one of these types; y, h: tensors to write (y may be x or residual, h the other
    or x: the stream's in-place update), else new ones. h of the result is what was
    normalised (None where y has taken the place of x without a residual: there is
    no backward pass then); mean and rstd are for the backward pass."""
    return LayerNorm(*_norm(x, weight, bias, residual, eps, y, h, stream, True))


def rms_norm(x, weight=None, residual=None, eps=1e-6, y=None, h=None, stream=None):
    """RMS norm of the rows of x, or of h = x + residual (meq_layer_norm); arguments as in layer_norm."""
    y, h, _, rstd = _norm(x, weight, None, residual, eps, y, h, stream, False)
    return RmsNorm(y, h, rstd)


def _norm_grad(dy, h, weight, mean, rstd, dh, dx, dweight, dbias, bias, stream):
    kind, shape, ld, device = _first(dy, "dy")
    if h is None:
        raise ValueError("h must be given: a norm whose y took the place of its x has none")
    rows, cols = shape
    dtype, where, f32 = dy.dtype, dy.device, _f32
    hp, ld_h = _matrix(h, dtype, shape, device, "h")
    sp, ld_s = _matrix(dh, dtype, shape, device, "dh")
    w, weight_kind = _columns(weight, cols, device, "weight")
    mp, rp = _vector(mean, f32, rows, device, "mean"), _vector(rstd, f32, rows, device, "rstd")
    given = [t for t in (dx, dweight, dbias) if t is not None]
    if dx is None:
        dx, ld_x = _memory(shape, dtype, where, stream), cols
        xp = dx.data_ptr()
    else:
        xp, ld_x = _matrix(dx, dtype, shape, device, "dx")
    like = dweight if dweight is not None else dbias if dbias is not None else weight  # of whose type both are
    grad_dtype, size = (f32, cols) if like is None else (like.dtype, like.shape)
    grad_kind, wp, bp = weight_kind if like is weight else _kind(like, "dweight"), None, None
    if dweight is not None:
        wp, _ = _columns(dweight, cols, device, "dweight")
    elif weight is not None:
        dweight = _memory(size, grad_dtype, where, stream)
        wp = dweight.data_ptr()
    if dbias is not None:
        bp, _ = _columns(dbias, cols, device, "dbias", grad_dtype)
    elif bias:
        dbias = _memory(size, grad_dtype, where, stream)
        bp = dbias.data_ptr()
    args = dy.data_ptr(), ld, hp, ld_h, sp, ld_s, kind, rows, cols, w, weight_kind, mp, rp, xp, ld_x, wp, bp, grad_kind
    # few elements mostly need no work: it is made where the call says so
    status = 1 if rows * cols > _FEW_ELEMENTS else lib.meq_layer_norm_grad(*args, None, _stream(stream, device))
    if status:
        work = _memory(_norm_work(rows, cols), f32, where, stream)
        _check_call(lib.meq_layer_norm_grad(*args, work.data_ptr(), _stream(stream, device)))
    if given:
        _increment(given)
    return dx, dweight, dbias


def layer_norm_grad(dy, h, weight, mean, rstd, dh=None, dx=None, dweight=None, dbias=None, bias=True, stream=None):
    """The backward pass of layer_norm (meq_layer_norm_grad) from the gradient dy
    of y and the h, mean and rstd of its result. dh: a gradient of h to add; dx,
    dweight, dbias: tensors to write (dx may be dy, h or dh), else new ones, of the
    weight's type; bias False: no bias. dx is the gradient of x and of the residual."""
    if mean is None:
        raise ValueError("mean must be given: without it the norm is rms_norm's")
    return LayerNormGrad(*_norm_grad(dy, h, weight, mean, rstd, dh, dx, dweight, dbias, bias, stream))


def rms_norm_grad(dy, h, weight, rstd, dh=None, dx=None, dweight=None, stream=None):
    """The backward pass of rms_norm (meq_layer_norm_grad); arguments as in layer_norm_grad."""
    dx, dweight, _ = _norm_grad(dy, h, weight, None, rstd, dh, dx, dweight, None, False, stream)
    return RmsNormGrad(dx, dweight)


def embedding(tokens, table, scale=1.0, out=None, dtype=None, stream=None):
    """scale times the table's rows of the tokens, one row per token
    (meq_embedding). tokens: contiguous int64 CUDA tensor, negative for rows of
    zeros; table: CUDA matrix, fp32, bf16 or fp16; out: the matrix to write, else a
    new one of dtype (default: the table's)."""
    table_kind, (vocab, cols), ld, device = _first(table, "table")
    n = tokens.numel()
    t = _vector(tokens, _i64, n, device, "tokens")
    given = out
    if out is None:
        out = _memory((n, cols), table.dtype if dtype is None else dtype, table.device, stream)
    elif dtype is not None and out.dtype is not dtype:
        raise ValueError(f"out must be of {dtype}")
    out_kind = _kind(out, "out")
    op, ld_out = _matrix(out, out.dtype, (n, cols), device, "out")
    _check_call(lib.meq_embedding(t, n, table.data_ptr(), table_kind, vocab, cols, ld, float(scale), op, out_kind, ld_out,
                                  _stream(stream, device)))
    if given is not None:
        _increment(given)
    return out


def embedding_grad(grad, tokens, out, scale=1.0, accumulate=False, stream=None):
    """The gradient of the table into out, a matrix of the table's shape
    (meq_embedding_grad), from the gradient of embedding's result. accumulate:
    added to what out holds. Returns out."""
    kind, (n, cols), ld, device = _first(grad, "grad")
    t = _vector(tokens, _i64, n, device, "tokens")
    out_kind = _kind(out, "out")
    vocab = out.shape[0]
    op, ld_out = _matrix(out, out.dtype, (vocab, cols), device, "out")
    work = _memory(lib.meq_embedding_work_floats(n, vocab, cols), _f32, grad.device, stream)
    _check_call(lib.meq_embedding_grad(grad.data_ptr(), kind, n, cols, ld, t, vocab, float(scale), op, out_kind, ld_out, bool(accumulate),
                                       work.data_ptr(), _stream(stream, device)))
    _increment(out)
    return out

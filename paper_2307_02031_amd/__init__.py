"""Python binding of libgbmw.so, the gfx950 library for the batched layer-wise
strategy search (Section 4.1.2, Eq. 3 and Appendix A of the paper).

The functions here have the names of the C entry points in include/gbmw.h and
only marshal arguments: every step of the search runs in the library's HIP
kernels.  There is no CPU fallback -- if the library has not been built
(``python paper_2307_02031_amd/build.py``) importing this package raises.

PyTorch is used for device memory and streams only: device-resident inputs are
torch CUDA tensors whose ``data_ptr()`` is handed to the library, and work is
enqueued on ``torch.cuda.current_stream()`` unless a stream is given.
"""
from __future__ import annotations

import collections.abc
import ctypes as ct
import functools
import operator
import os
import struct

import numpy as np
import torch  # imported first so that the library binds to the same HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgbmw.so")

GBMW_OK, GBMW_ERR_INVALID_ARG, GBMW_ERR_UNSUPPORTED, GBMW_ERR_OOM, GBMW_ERR_DEVICE = range(5)
GBMW_PTR_HOST, GBMW_PTR_DEVICE = 0, 1
GBMW_FLAG_KEEP_ALL_C = 1
GBMW_FLAG_TIME_KERNELS = 2
GBMW_FLAG_ONE_STREAM = 4
GBMW_FLAG_RESOLVE_ALL = 8
GBMW_FLAG_LAZY_ARGMIN = 16
GBMW_FLAG_DENSE_ARITHMETIC = 32
GBMW_FLAG_COUNT_WORK = 64
GBMW_FLAG_LAYER_LAUNCHES = 128
GBMW_FLAG_TEST_WAIT_GIVES_UP = 256
GBMW_FLAG_COOPERATIVE_LAUNCH = 512
GBMW_MAX_S = 256
GBMW_STATIC_SCRATCH_BYTES = 1 << 20

EXPORTS = [
    "gbmw_dp_solve_batched", "gbmw_backtrack", "gbmw_backtrack_static", "gbmw_select_forward_budget", "gbmw_pipeline_cost",
    "gbmw_partition_search", "gbmw_enumerate_strategies", "gbmw_cost_model",
    "gbmw_attention_forward", "gbmw_attention_backward", "gbmw_attention_workspace",
    "gbmw_layer_norm_forward", "gbmw_layer_norm_backward", "gbmw_layer_norm_workspace",
    "gbmw_gradient_list_create", "gbmw_clip_gradients", "gbmw_gradient_list_destroy",
    "gbmw_rms_norm_forward", "gbmw_rms_norm_backward", "gbmw_rms_norm_workspace",
    "gbmw_rotary_forward", "gbmw_rotary_backward", "gbmw_rotary_frequencies",
    "gbmw_adamw_list_create", "gbmw_adamw_step", "gbmw_adamw_list_destroy",
    "gbmw_max_layers", "gbmw_get_best",
    "gbmw_export_tables", "gbmw_synchronize", "gbmw_last_solve_ms", "gbmw_last_solve_work", "gbmw_destroy",
    "gbmw_last_error", "gbmw_version",
]


class gbmw_problem(ct.Structure):
    _fields_ = [("B", ct.c_int32), ("S", ct.c_int32), ("E", ct.c_int32),
                ("L", ct.c_void_p), ("c", ct.c_void_p), ("M", ct.c_void_p), ("R", ct.c_void_p),
                ("ptr_space", ct.c_int32), ("stream", ct.c_void_p)]


class gbmw_partition_problem(ct.Structure):
    _fields_ = [("n_chain", ct.c_int32), ("S", ct.c_int32), ("E", ct.c_int32), ("max_iter", ct.c_int32),
                ("P", ct.c_void_p), ("Lm", ct.c_void_p), ("m", ct.c_void_p), ("c", ct.c_void_p),
                ("c_nosync", ct.c_void_p), ("R", ct.c_void_p), ("M", ct.c_void_p), ("p0", ct.c_void_p),
                ("p_t", ct.c_void_p), ("stream", ct.c_void_p), ("batch_size", ct.c_void_p),
                ("batch_group", ct.c_void_p), ("O_b", ct.c_void_p), ("O_ms", ct.c_void_p)]


class gbmw_partition_result(ct.Structure):
    _fields_ = [("n_iter", ct.c_void_p), ("O_t", ct.c_void_p), ("p", ct.c_void_p), ("cost", ct.c_void_p),
                ("C", ct.c_void_p), ("Cns", ct.c_void_p), ("O", ct.c_void_p), ("alpha_t", ct.c_void_p),
                ("alpha_m", ct.c_void_p), ("strat", ct.c_void_p),
                ("rounds", ct.c_int32), ("stage_solves", ct.c_int32), ("cell_updates", ct.c_int64),
                ("device_ms", ct.c_float), ("tpt", ct.c_float), ("tpt_group", ct.c_int32),
                ("tpt_pair", ct.c_int32)]


class gbmw_strategy(ct.Structure):
    _fields_ = [("n_levels", ct.c_int32), ("kind", ct.c_int32 * 3), ("degree", ct.c_int32 * 3), ("ckpt", ct.c_int32)]


class gbmw_hardware(ct.Structure):
    _fields_ = [("rate", ct.c_double), ("bw_in", ct.c_double), ("bw_out", ct.c_double),
                ("param_bytes", ct.c_double), ("state_bytes", ct.c_double), ("slow", ct.c_double),
                ("unit_bytes", ct.c_double), ("island", ct.c_int32)]


GBMW_F32, GBMW_F16, GBMW_BF16 = 0, 1, 2
GBMW_E4M3, GBMW_I8 = 3, 4
GBMW_ROTARY_NONE, GBMW_ROTARY_LINEAR, GBMW_ROTARY_BASE, GBMW_ROTARY_RAMP = range(4)


class gbmw_attention_problem(ct.Structure):
    _fields_ = ([(n, ct.c_int32) for n in ("dtype", "B", "Hq", "Hk", "Lq", "Lk", "D", "causal")] +
                [("scale", ct.c_float)] +
                [(n, ct.c_void_p) for n in ("len_q", "len_k", "q", "k", "v")] +
                [(n, ct.c_int64 * 3) for n in ("q_stride", "k_stride", "v_stride")] +
                [("out", ct.c_void_p), ("out_stride", ct.c_int64 * 3), ("lse", ct.c_void_p),
                 ("dout", ct.c_void_p), ("dout_stride", ct.c_int64 * 3)] +
                [(n, ct.c_void_p) for n in ("dq", "dk", "dv")] +
                [(n, ct.c_int64 * 3) for n in ("dq_stride", "dk_stride", "dv_stride")] +
                [("workspace", ct.c_void_p), ("workspace_bytes", ct.c_int64), ("stream", ct.c_void_p)])


class gbmw_layer_norm_problem(ct.Structure):
    _fields_ = [("dtype", ct.c_int32), ("wdtype", ct.c_int32), ("rows", ct.c_int64), ("cols", ct.c_int32),
                ("eps", ct.c_float), ("x", ct.c_void_p), ("x_stride", ct.c_int64), ("weight", ct.c_void_p),
                ("bias", ct.c_void_p), ("y", ct.c_void_p), ("y_stride", ct.c_int64), ("mean", ct.c_void_p),
                ("rstd", ct.c_void_p), ("dy", ct.c_void_p), ("dy_stride", ct.c_int64), ("dx", ct.c_void_p),
                ("dx_stride", ct.c_int64), ("dweight", ct.c_void_p), ("dbias", ct.c_void_p),
                ("workspace", ct.c_void_p), ("workspace_bytes", ct.c_int64), ("stream", ct.c_void_p)]


class gbmw_rms_norm_problem(ct.Structure):
    _fields_ = ([("dtype", ct.c_int32), ("wdtype", ct.c_int32), ("rows", ct.c_int64), ("cols", ct.c_int32),
                 ("eps", ct.c_float), ("x", ct.c_void_p), ("x_stride", ct.c_int64), ("weight", ct.c_void_p),
                 ("rstd", ct.c_void_p)] +
                [f for n in ("residual", "h", "y", "q") for f in ((n, ct.c_void_p), (n + "_stride", ct.c_int64))] +
                [("scale", ct.c_void_p), ("qtype", ct.c_int32), ("group", ct.c_int32)] +
                [f for n in ("dy", "dres", "dx") for f in ((n, ct.c_void_p), (n + "_stride", ct.c_int64))] +
                [("dweight", ct.c_void_p), ("workspace", ct.c_void_p), ("workspace_bytes", ct.c_int64),
                 ("stream", ct.c_void_p)])


class gbmw_rotary_problem(ct.Structure):
    _fields_ = ([(n, ct.c_int32) for n in ("dtype", "B", "L", "Hq", "Hk", "D", "rot", "interleaved")] +
                [("factor", ct.c_float), ("freq", ct.c_void_p), ("positions", ct.c_void_p),
                 ("position_stride", ct.c_int64), ("len", ct.c_void_p), ("q", ct.c_void_p), ("k", ct.c_void_p),
                 ("q_stride", ct.c_int64 * 3), ("k_stride", ct.c_int64 * 3), ("q_out", ct.c_void_p),
                 ("k_out", ct.c_void_p), ("q_out_stride", ct.c_int64 * 3), ("k_out_stride", ct.c_int64 * 3),
                 ("stream", ct.c_void_p)])


# the same, packed at once: filling a structure's arrays of strides one by one takes 2.5 us longer
_ROTARY = struct.Struct("@8if4xQQqQQQ6qQQ6qQ")
assert _ROTARY.size == ct.sizeof(gbmw_rotary_problem)


class gbmw_adamw_tensor(ct.Structure):
    _fields_ = ([("numel", ct.c_int64)] +
                [(n, ct.c_void_p) for n in ("grad", "param", "copy", "m", "v", "m_scale", "v_scale")] +
                [(n, ct.c_int32) for n in ("grad_dtype", "dtype", "copy_dtype")] + [("weight_decay", ct.c_float)])


class gbmw_adamw_options(ct.Structure):
    _fields_ = ([(n, ct.c_double) for n in ("lr", "beta1", "beta2", "eps", "scale", "max_norm")] +
                [("step", ct.c_int64), ("seed", ct.c_uint32)] +
                [(n, ct.c_void_p) for n in ("norm", "lr_now", "step_now")])


STRATEGY_DTYPE = np.dtype([("n_levels", np.int32), ("kind", np.int32, 3), ("degree", np.int32, 3), ("ckpt", np.int32)])
GBMW_DP, GBMW_SDP, GBMW_TP = 1, 2, 3


class GbmwError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gbmw status {status}: {message}")
        self.status = status


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2307_02031_amd/build.py` "
                      "(there is no CPU fallback)")
_lib = ct.CDLL(LIB_PATH)
_lib.gbmw_dp_solve_batched.argtypes = [ct.POINTER(gbmw_problem), ct.c_uint32, ct.POINTER(ct.c_void_p)]
_lib.gbmw_dp_solve_batched.restype = ct.c_int
_lib.gbmw_backtrack.argtypes = [ct.c_void_p, ct.c_int32] + [ct.c_void_p] * 5
_lib.gbmw_backtrack.restype = ct.c_int
_lib.gbmw_backtrack_static.argtypes = [ct.c_void_p, ct.c_int32] + [ct.c_void_p] * 5
_lib.gbmw_backtrack_static.restype = ct.c_int
_lib.gbmw_select_forward_budget.argtypes = [ct.c_void_p] * 8
_lib.gbmw_select_forward_budget.restype = ct.c_int
_lib.gbmw_pipeline_cost.argtypes = [ct.c_void_p, ct.c_int32] + [ct.c_void_p] * 8
_lib.gbmw_pipeline_cost.restype = ct.c_int
_lib.gbmw_partition_search.argtypes = [ct.POINTER(gbmw_partition_problem), ct.c_uint32,
                                       ct.POINTER(gbmw_partition_result), ct.POINTER(ct.c_void_p)]
_lib.gbmw_partition_search.restype = ct.c_int
_lib.gbmw_enumerate_strategies.argtypes = [ct.c_int32, ct.c_int32, ct.c_int32, ct.c_void_p, ct.c_int32]
_lib.gbmw_enumerate_strategies.restype = ct.c_int32
for _name in ("gbmw_attention_forward", "gbmw_attention_backward"):
    getattr(_lib, _name).argtypes = [ct.POINTER(gbmw_attention_problem)]
    getattr(_lib, _name).restype = ct.c_int
_lib.gbmw_attention_workspace.argtypes = [ct.POINTER(gbmw_attention_problem), ct.c_int32]
_lib.gbmw_attention_workspace.restype = ct.c_int64
for _name in ("gbmw_layer_norm_forward", "gbmw_layer_norm_backward"):
    getattr(_lib, _name).argtypes = [ct.POINTER(gbmw_layer_norm_problem)]
    getattr(_lib, _name).restype = ct.c_int
_lib.gbmw_layer_norm_workspace.argtypes = [ct.POINTER(gbmw_layer_norm_problem)]
_lib.gbmw_layer_norm_workspace.restype = ct.c_int64
_lib.gbmw_gradient_list_create.argtypes = [ct.c_int32] + [ct.c_void_p] * 5 + [ct.POINTER(ct.c_void_p)]
_lib.gbmw_gradient_list_create.restype = ct.c_int
_lib.gbmw_clip_gradients.argtypes = [ct.c_void_p, ct.c_float, ct.c_float, ct.c_void_p, ct.c_void_p]
_lib.gbmw_clip_gradients.restype = ct.c_int
_lib.gbmw_gradient_list_destroy.argtypes = [ct.c_void_p]
_lib.gbmw_gradient_list_destroy.restype = None
for _name in ("gbmw_rms_norm_forward", "gbmw_rms_norm_backward", "gbmw_rms_norm_workspace"):
    getattr(_lib, _name).argtypes = [ct.POINTER(gbmw_rms_norm_problem)]
    getattr(_lib, _name).restype = ct.c_int64 if _name.endswith("workspace") else ct.c_int
for _name in ("gbmw_rotary_forward", "gbmw_rotary_backward"):
    getattr(_lib, _name).argtypes = [ct.POINTER(gbmw_rotary_problem)]
    getattr(_lib, _name).restype = ct.c_int
_lib.gbmw_rotary_frequencies.argtypes = [ct.c_int32, ct.c_double, ct.c_int32] + [ct.c_double] * 4 + [ct.c_void_p]
_lib.gbmw_rotary_frequencies.restype = ct.c_int
_lib.gbmw_adamw_list_create.argtypes = [ct.c_int32, ct.POINTER(gbmw_adamw_tensor), ct.c_int32, ct.POINTER(ct.c_void_p)]
_lib.gbmw_adamw_list_create.restype = ct.c_int
_lib.gbmw_adamw_step.argtypes = [ct.c_void_p, ct.POINTER(gbmw_adamw_options), ct.c_void_p]
_lib.gbmw_adamw_step.restype = ct.c_int
_lib.gbmw_adamw_list_destroy.argtypes = [ct.c_void_p]
_lib.gbmw_adamw_list_destroy.restype = None
_lib.gbmw_cost_model.argtypes = [ct.c_void_p, ct.c_int32, ct.c_void_p, ct.c_int32, ct.POINTER(gbmw_hardware),
                                 ct.c_double, ct.c_int32, ct.c_int32] + [ct.c_void_p] * 8
_lib.gbmw_cost_model.restype = ct.c_int
_lib.gbmw_max_layers.argtypes = [ct.c_void_p]
_lib.gbmw_max_layers.restype = ct.c_int32
_lib.gbmw_get_best.argtypes = [ct.c_void_p, ct.c_void_p, ct.c_void_p]
_lib.gbmw_get_best.restype = ct.c_int
_lib.gbmw_export_tables.argtypes = [ct.c_void_p, ct.c_int32, ct.c_int32, ct.c_int32, ct.c_void_p, ct.c_void_p]
_lib.gbmw_export_tables.restype = ct.c_int
_lib.gbmw_synchronize.argtypes = [ct.c_void_p]
_lib.gbmw_synchronize.restype = ct.c_int
_lib.gbmw_last_solve_ms.argtypes = [ct.c_void_p, ct.POINTER(ct.c_float), ct.POINTER(ct.c_float),
                                    ct.POINTER(ct.c_int32)]
_lib.gbmw_last_solve_ms.restype = ct.c_int
_lib.gbmw_last_solve_work.argtypes = [ct.c_void_p, ct.c_int32, ct.POINTER(ct.c_uint64)]
_lib.gbmw_last_solve_work.restype = ct.c_int
_lib.gbmw_destroy.argtypes = [ct.c_void_p]
_lib.gbmw_destroy.restype = None
_lib.gbmw_last_error.restype = ct.c_char_p
_lib.gbmw_version.restype = ct.c_char_p


def gbmw_last_error() -> str:
    return _lib.gbmw_last_error().decode()


def gbmw_version() -> str:
    return _lib.gbmw_version().decode()


def _check(status: int):
    if status != GBMW_OK:
        raise GbmwError(status, gbmw_last_error())


class Context:
    """Owner of a gbmw_ctx*; keeps the arrays handed to the library alive."""

    def __init__(self):
        self.handle = ct.c_void_p(None)
        self.B = self.S = self.E = 0
        self.L = None
        self._keep = ()

    def __del__(self):
        try:
            gbmw_destroy(self)
        except Exception:
            pass


def _ptr(a):
    if isinstance(a, torch.Tensor):
        return a.data_ptr()
    return a.ctypes.data


def gbmw_dp_solve_batched(L, c, M, R, S: int, E: int, flags: int = 0, ctx: Context | None = None,
                          stream: int | None = None) -> Context:
    """Enqueue the table fill for B = len(L) instances.

    c [sumL][S] f32, M [sumL][S] i32, R [sumL][S][S] f32: either all numpy
    arrays (host) or all torch CUDA tensors (device, used in place).  Returns
    the context (a new one unless ``ctx`` is given)."""
    L = np.ascontiguousarray(L, dtype=np.int32)
    on_dev = isinstance(c, torch.Tensor)
    if on_dev:
        assert all(isinstance(x, torch.Tensor) and x.is_cuda and x.is_contiguous() for x in (c, M, R))
        assert c.dtype == torch.float32 and M.dtype == torch.int32 and R.dtype == torch.float32
    else:
        c = np.ascontiguousarray(c, dtype=np.float32)
        M = np.ascontiguousarray(M, dtype=np.int32)
        R = np.ascontiguousarray(R, dtype=np.float32)
    sumL = int(L.sum())
    assert tuple(c.shape) == (sumL, S) and tuple(M.shape) == (sumL, S) and tuple(R.shape) == (sumL, S, S)
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    p = gbmw_problem(len(L), S, E, L.ctypes.data, _ptr(c), _ptr(M), _ptr(R),
                     GBMW_PTR_DEVICE if on_dev else GBMW_PTR_HOST, stream)
    if ctx is None:
        ctx = Context()
    _check(_lib.gbmw_dp_solve_batched(ct.byref(p), flags, ct.byref(ctx.handle)))
    ctx.B, ctx.S, ctx.E, ctx.L = len(L), S, E, L
    ctx._keep = (L, c, M, R)
    return ctx


def gbmw_synchronize(ctx: Context) -> None:
    _check(_lib.gbmw_synchronize(ctx.handle))


def gbmw_max_layers(ctx: Context) -> int:
    return int(_lib.gbmw_max_layers(ctx.handle))


def gbmw_get_best(ctx: Context):
    """best [B][E+1] float32, best_s [B][E+1] uint8 (host arrays)."""
    best = np.empty((ctx.B, ctx.E + 1), np.float32)
    best_s = np.empty((ctx.B, ctx.E + 1), np.uint8)
    _check(_lib.gbmw_get_best(ctx.handle, best.ctypes.data, best_s.ctypes.data))
    return best, best_s


def gbmw_backtrack(ctx: Context, q_instance, q_e):
    """plan [nq][Lmax] uint8 (0xFF padded), cost [nq] float32, mem_used [nq] int32."""
    qi = np.ascontiguousarray(q_instance, dtype=np.int32)
    qe = np.ascontiguousarray(q_e, dtype=np.int32)
    assert qi.shape == qe.shape and qi.ndim == 1
    nq, Lmax = len(qi), gbmw_max_layers(ctx)
    plan = np.empty((nq, Lmax), np.uint8)
    cost = np.empty(nq, np.float32)
    mem = np.empty(nq, np.int32)
    _check(_lib.gbmw_backtrack(ctx.handle, nq, qi.ctypes.data, qe.ctypes.data, plan.ctypes.data,
                               cost.ctypes.data, mem.ctypes.data))
    return plan, cost, mem


def gbmw_backtrack_static(ctx: Context, q_instance, q_e):
    """gbmw_backtrack through the library's fixed staging block (no device allocation)."""
    qi = np.ascontiguousarray(q_instance, dtype=np.int32)
    qe = np.ascontiguousarray(q_e, dtype=np.int32)
    assert qi.shape == qe.shape and qi.ndim == 1
    nq, Lmax = len(qi), gbmw_max_layers(ctx)
    plan = np.empty((nq, Lmax), np.uint8)
    cost = np.empty(nq, np.float32)
    mem = np.empty(nq, np.int32)
    _check(_lib.gbmw_backtrack_static(ctx.handle, nq, qi.ctypes.data, qe.ctypes.data, plan.ctypes.data,
                                      cost.ctypes.data, mem.ctypes.data))
    return plan, cost, mem


def gbmw_select_forward_budget(ctx: Context, O_f, O_b, O_ms):
    """Algorithm 3's outer loop: e_opt [B] int32, cost [B] float32, plan [B][Lmax] uint8,
    e_all [B] int32 (host arrays)."""
    sumL = int(ctx.L.sum())
    arrs = [np.ascontiguousarray(a, dtype=np.int32) for a in (O_f, O_b, O_ms)]
    assert all(a.shape == (sumL, ctx.S) for a in arrs)
    Lmax = gbmw_max_layers(ctx)
    e_opt = np.empty(ctx.B, np.int32)
    cost = np.empty(ctx.B, np.float32)
    plan = np.empty((ctx.B, Lmax), np.uint8)
    e_all = np.empty(ctx.B, np.int32)
    _check(_lib.gbmw_select_forward_budget(ctx.handle, arrs[0].ctypes.data, arrs[1].ctypes.data,
                                           arrs[2].ctypes.data, e_opt.ctypes.data, cost.ctypes.data,
                                           plan.ctypes.data, e_all.ctypes.data))
    return e_opt, cost, plan, e_all


def gbmw_pipeline_cost(ctx: Context, stage_begin, stage_instance, stage_e, microbatches, c_nosync=None):
    """Eq. 5 / Eq. 8: cost [n_pipe], stage_cost [n_stage], stage_cost_nosync [n_stage] (float32)."""
    sb = np.ascontiguousarray(stage_begin, dtype=np.int32)
    si = np.ascontiguousarray(stage_instance, dtype=np.int32)
    se = np.ascontiguousarray(stage_e, dtype=np.int32)
    mb = np.ascontiguousarray(microbatches, dtype=np.int32)
    n_pipe = len(mb)
    assert sb.shape == (n_pipe + 1,) and si.shape == se.shape == (int(sb[-1]),)
    cns = None if c_nosync is None else np.ascontiguousarray(c_nosync, dtype=np.float32)
    if cns is not None:
        assert cns.shape == (int(ctx.L.sum()), ctx.S)
    cost = np.empty(n_pipe, np.float32)
    sc = np.empty(len(si), np.float32)
    scn = np.empty(len(si), np.float32)
    _check(_lib.gbmw_pipeline_cost(ctx.handle, n_pipe, sb.ctypes.data, si.ctypes.data, se.ctypes.data,
                                   mb.ctypes.data, None if cns is None else cns.ctypes.data,
                                   cost.ctypes.data, sc.ctypes.data, scn.ctypes.data))
    return cost, sc, scn


def gbmw_partition_search(P, Lm, m, c, c_nosync, R, M, p0, p_t, S: int, E: int, max_iter: int = 64,
                          flags: int = 0, ctx: Context | None = None, stream: int | None = None,
                          batch_size=None, batch_group=None, O_b=None, O_ms=None):
    """Algorithm 2's inner loop for n_chain = len(P) pairs (host numpy arrays, the
    pairs' rows concatenated; c_nosync and p_t may be None; O_b and O_ms, shaped like M,
    switch the stage searches to Appendix A's forward-budget selection).  Returns (result dict,
    ctx): n_iter, O_t [n]; p, C, Cns, O [n][max_iter][Pmax]; cost, alpha_t, alpha_m
    [n][max_iter]; strat [n][Lmmax]; rounds, stage_solves, cell_updates, device_ms."""
    i32 = lambda a: None if a is None else np.ascontiguousarray(a, dtype=np.int32)
    f32 = lambda a: None if a is None else np.ascontiguousarray(a, dtype=np.float32)
    P, Lm, m, M, p0, p_t = (i32(a) for a in (P, Lm, m, M, p0, p_t))
    c, c_nosync, R, batch_size = (f32(a) for a in (c, c_nosync, R, batch_size))
    batch_group, O_b, O_ms = i32(batch_group), i32(O_b), i32(O_ms)
    n, sumLm, sumP = len(P), int(Lm.sum()), int(P.sum())
    sumPL = int((P.astype(np.int64) * Lm).sum())
    assert Lm.shape == m.shape == (n,) and c.shape == (sumLm, S) and R.shape == (sumLm, S, S)
    assert M.shape == (sumPL, S) and p0.shape == (sumP,)
    assert c_nosync is None or c_nosync.shape == c.shape
    assert p_t is None or p_t.shape == p0.shape
    assert (O_b is None or O_b.shape == M.shape) and (O_ms is None or O_ms.shape == M.shape)
    Pmax, Lmmax = int(P.max()), int(Lm.max())
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    ptr = lambda a: None if a is None else a.ctypes.data
    q = gbmw_partition_problem(n, S, E, max_iter, ptr(P), ptr(Lm), ptr(m), ptr(c), ptr(c_nosync), ptr(R),
                               ptr(M), ptr(p0), ptr(p_t), stream, ptr(batch_size), ptr(batch_group),
                               ptr(O_b), ptr(O_ms))
    mi = max(1, max_iter)
    res = dict(n_iter=np.zeros(n, np.int32), O_t=np.zeros(n, np.int32),
               p=np.zeros((n, mi, Pmax), np.int32), cost=np.zeros((n, mi), np.float32),
               C=np.zeros((n, mi, Pmax), np.float32), Cns=np.zeros((n, mi, Pmax), np.float32),
               O=np.zeros((n, mi, Pmax), np.int32), alpha_t=np.zeros((n, mi), np.float32),
               alpha_m=np.zeros((n, mi), np.float32), strat=np.zeros((n, Lmmax), np.uint8))
    out = gbmw_partition_result(*[res[k].ctypes.data for k in ("n_iter", "O_t", "p", "cost", "C", "Cns", "O",
                                                               "alpha_t", "alpha_m", "strat")], 0, 0, 0, 0.0, 0.0, -1, -1)
    if ctx is None:
        ctx = Context()
    _check(_lib.gbmw_partition_search(ct.byref(q), flags, ct.byref(out), ct.byref(ctx.handle)))
    ctx.B = ctx.S = ctx.E = 0
    ctx.L, ctx._keep = None, ()
    res.update(rounds=out.rounds, stage_solves=out.stage_solves, cell_updates=out.cell_updates,
               device_ms=out.device_ms, tpt=np.float32(out.tpt), tpt_group=out.tpt_group, tpt_pair=out.tpt_pair)
    return res, ctx


def gbmw_enumerate_strategies(group_size: int, with_ckpt: bool = True, takeaway3: bool = True) -> np.ndarray:
    """Structured array (STRATEGY_DTYPE) of the candidate strategies of one layer."""
    n = _lib.gbmw_enumerate_strategies(group_size, int(with_ckpt), int(takeaway3), None, 0)
    if n < 0:
        raise GbmwError(GBMW_ERR_INVALID_ARG, gbmw_last_error())
    out = np.zeros(n, STRATEGY_DTYPE)
    assert STRATEGY_DTYPE.itemsize == ct.sizeof(gbmw_strategy)
    _lib.gbmw_enumerate_strategies(group_size, int(with_ckpt), int(takeaway3), out.ctypes.data, n)
    return out


def gbmw_cost_model(layers, strategies, hw: dict, Bm: float, P: int, device: bool = False,
                    stream: int | None = None) -> dict:
    """c, c_nosync [L][S] f32; O_f, O_b, O_ms [L][S] i32; M [P][L][S] i32; R [L][S][S] f32 --
    numpy arrays, or torch CUDA tensors if ``device``.  layers: float64 [L][4] (params,
    flops, bnd, intm); strategies: STRATEGY_DTYPE array."""
    layers = np.ascontiguousarray(layers, dtype=np.float64)
    strategies = np.ascontiguousarray(strategies, dtype=STRATEGY_DTYPE)
    L, S = len(layers), len(strategies)
    assert layers.shape == (L, 4)
    h = gbmw_hardware(hw["rate"], hw["bw_in"], hw["bw_out"], hw["param_bytes"], hw["state_bytes"], hw["slow"],
                      hw["unit_bytes"], hw["island"])
    shapes = dict(c=((L, S), np.float32), c_nosync=((L, S), np.float32), O_f=((L, S), np.int32),
                  O_b=((L, S), np.int32), O_ms=((L, S), np.int32), M=((P, L, S), np.int32), R=((L, S, S), np.float32))
    if device:
        tdt = {np.float32: torch.float32, np.int32: torch.int32}
        out = {k: torch.empty(sh, dtype=tdt[dt], device="cuda") for k, (sh, dt) in shapes.items()}
    else:
        out = {k: np.empty(sh, dt) for k, (sh, dt) in shapes.items()}
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    _check(_lib.gbmw_cost_model(layers.ctypes.data, L, strategies.ctypes.data, S, ct.byref(h), float(Bm), P,
                                GBMW_PTR_DEVICE if device else GBMW_PTR_HOST,
                                *[_ptr(out[k]) for k in ("c", "c_nosync", "O_f", "O_b", "O_ms", "M", "R")], stream))
    return out


# ---- operators of a transformer layer's training ------------------------------------------------------------------
#
# torch's autograd does not record these calls: results carry no graph, also of tensors that require grad, and the
# backward calls are the caller's to make (in a torch.autograd.Function, or by hand as in layer_example).

_DTYPE = {torch.float32: GBMW_F32, torch.float16: GBMW_F16, torch.bfloat16: GBMW_BF16}


def _refuse(message: str):
    raise GbmwError(GBMW_ERR_INVALID_ARG, message)


# the current device and the current stream's handle without checks and objects around them, where torch has them
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _refuse_tensor(name: str, t, device: int, dtype, shape):
    """Says what is wrong with t: the kernels take plain addresses, so type, place and shape are checked here."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} is not a tensor on the GPU")
    if t.get_device() != device:
        _refuse(f"{name} is on {t.device}, device {device} is current")
    if t.dtype != dtype:
        _refuse(f"{name} has type {t.dtype}, not {dtype}")
    _refuse(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _check_tensor(name: str, t, device: int, dtype, shape) -> None:
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype != dtype or t.shape != shape:
        _refuse_tensor(name, t, device, dtype, shape)


def _check_counts(name: str, sizes: int) -> None:
    """sizes: the sizes' bits together.  What the library counts in 32 bits would lose its upper ones without a word."""
    if sizes >> 31:
        _refuse(f"{name}: a size of 2^31 or more")


def _device_of(name: str, t, types) -> int:
    """The current device, which the first argument has to be on, with one of the types."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} is not a tensor on the GPU")
    device = _current_device()
    if t.get_device() != device:
        _refuse(f"{name} is on {t.device}, device {device} is current")
    if t.dtype not in types:
        _refuse(f"{name} has type {t.dtype}")
    return device


def _stream_of(stream):
    """A torch stream for one, or for a handle.  0 is the default stream's: an ExternalStream of it would be a new
    stream, which waits for nobody."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = int(getattr(stream, "cuda_stream", stream))
    return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()


def _on_stream(call):
    """call with one more argument: `stream`, a torch stream or a handle, by default the current one.  Outputs and
    scratch memory that a call makes belong to the stream its kernels run on, so that the memory is not handed to
    anybody else before they have run.  Inputs on another stream than that are the caller's to keep until the stream
    has got to the call, as with any work on a second stream."""
    @functools.wraps(call)
    def on_stream(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(_stream_of(stream)):
            return call(*args, **kw)
    return on_stream


def _workspace(p, given, need: int, device: int):
    """Sets p's workspace: the caller's uint8 tensor, or a new one.  Returns what has to live until the call is made."""
    if need < 0:
        raise GbmwError(GBMW_ERR_INVALID_ARG, gbmw_last_error())
    if given is None:
        given = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    elif not isinstance(given, torch.Tensor) or given.get_device() != device or given.dtype != torch.uint8 \
            or not given.is_contiguous():
        _refuse("workspace is not a contiguous uint8 tensor on the current GPU")
    p.workspace, p.workspace_bytes = given.data_ptr(), given.numel()
    return given


def _strides(name: str, t) -> tuple:
    s0, s1, s2, s3 = t.stride()
    if s3 != 1 and t.shape[3] > 1:
        _refuse(f"{name}: the values of one head are not next to each other")
    return s0, s1, s2


def _set_array(p, name: str, t) -> None:
    setattr(p, name, t.data_ptr())
    setattr(p, name + "_stride", _strides(name, t))


_HALF_TYPES = (torch.bfloat16, torch.float16, torch.float32)      # float32: the library says that it is not supported


def _attention_problem(q, k, v, causal, scale, len_q, len_k):
    device = _device_of("q", q, _HALF_TYPES)
    shape, dtype = q.shape, q.dtype
    if len(shape) != 4:
        _refuse(f"q has {q.dim()} dimensions, not [B][Lq][Hq][D]")
    if not isinstance(k, torch.Tensor) or k.dim() != 4:
        _refuse("k is not a tensor [B][Lk][Hk][D]")
    B, Lq, Hq, D = shape
    kshape = k.shape
    if kshape[0] != B or kshape[3] != D or k.dtype != dtype or k.get_device() != device:
        _refuse_tensor("k", k, device, dtype, (B, kshape[1], kshape[2], D))
    _check_tensor("v", v, device, dtype, kshape)
    _check_counts("q and k", B | Lq | Hq | D | kshape[1] | kshape[2])
    if len_q is not None:
        len_q = _length("len_q", len_q, device, B)
    if len_k is not None:
        len_k = _length("len_k", len_k, device, B)
    p = gbmw_attention_problem(_DTYPE[dtype], B, Hq, kshape[2], Lq, kshape[1], D, 1 if causal else 0,
                               (1.0 / D ** 0.5 if D else 1.0) if scale is None else scale, len_q, len_k,
                               q.data_ptr(), k.data_ptr(), v.data_ptr(),
                               _strides("q", q), _strides("k", k), _strides("v", v))
    p.stream = _raw_stream(device)
    return p, device


def _length(name: str, t, device: int, B: int) -> int:
    _check_tensor(name, t, device, torch.int32, (B,))
    if not t.is_contiguous():
        _refuse(f"{name} is not contiguous")
    return t.data_ptr()


def _lse(p, lse, device: int) -> None:
    _check_tensor("lse", lse, device, torch.float32, (p.B, p.Hq, p.Lq))
    if not lse.is_contiguous():
        _refuse("lse is not contiguous")
    p.lse = lse.data_ptr()


def gbmw_attention_workspace(q, k, backward: bool, causal: bool | None = None) -> int:
    """Bytes of workspace of a call on q [B][Lq][Hq][D] and k [B][Lk][Hk][D].  causal: the call's mask; by default as
    many bytes as either mask needs."""
    _check_counts("q and k", functools.reduce(operator.or_, (*q.shape, *k.shape)))
    p = gbmw_attention_problem()
    p.dtype, (p.B, p.Lq, p.Hq, p.D), (p.Lk, p.Hk) = _DTYPE.get(q.dtype, -1), q.shape, (k.shape[1], k.shape[2])
    need = 0
    for p.causal in (0, 1) if causal is None else (1 if causal else 0,):
        n = _lib.gbmw_attention_workspace(ct.byref(p), int(backward))
        if n < 0:
            raise GbmwError(GBMW_ERR_INVALID_ARG, gbmw_last_error())
        need = max(need, n)
    return need


def _new_like(t, dtype=None):
    """A dense tensor like t, of t's type or another."""
    return torch.empty_like(t, dtype=dtype) if t.is_contiguous() else torch.empty(t.shape, dtype=dtype or t.dtype, device="cuda")


@_on_stream
def gbmw_attention_forward(q, k, v, causal: bool = False, scale: float | None = None, len_q=None, len_k=None,
                           out=None, lse=None, workspace=None):
    """out [B][Lq][Hq][D] and lse [B][Hq][Lq] (float32) of q [B][Lq][Hq][D], k and v [B][Lk][Hk][D]: float16 or
    bfloat16 GPU tensors with any strides whose last one is 1.  scale: 1 / sqrt(D) by default.  len_q, len_k:
    int32 [B], the samples' lengths.  out, lse, workspace (uint8): made here unless given.  stream=: as everywhere.
    Not recorded by autograd: gradients come from gbmw_attention_backward."""
    p, device = _attention_problem(q, k, v, causal, scale, len_q, len_k)
    if out is None:
        out = _new_like(q)
    else:
        _check_tensor("out", out, device, q.dtype, q.shape)
    if lse is None:
        lse = torch.empty((p.B, p.Hq, p.Lq), dtype=torch.float32, device="cuda")
        p.lse = lse.data_ptr()
    else:
        _lse(p, lse, device)
    _set_array(p, "out", out)
    ref = ct.byref(p)
    need = _lib.gbmw_attention_workspace(ref, 0)
    keep = _workspace(p, workspace, need, device) if need else None
    _check(_lib.gbmw_attention_forward(ref))
    return out, lse


@_on_stream
def gbmw_attention_backward(dout, q, k, v, out, lse, causal: bool = False, scale: float | None = None, len_q=None,
                            len_k=None, dq=None, dk=None, dv=None, workspace=None):
    """dq, dk, dv from dout and the forward call's arguments and results, all of its keys: a call on a part of the keys
    with out and lse of all of them gives something else.  stream=: as everywhere."""
    p, device = _attention_problem(q, k, v, causal, scale, len_q, len_k)
    dtype, qshape, kshape = q.dtype, q.shape, k.shape
    _check_tensor("dout", dout, device, dtype, qshape)
    _check_tensor("out", out, device, dtype, qshape)
    _lse(p, lse, device)
    if dq is None:
        dq = _new_like(q)
    else:
        _check_tensor("dq", dq, device, dtype, qshape)
    if dk is None:
        dk = _new_like(k)
    else:
        _check_tensor("dk", dk, device, dtype, kshape)
    if dv is None:
        dv = torch.empty_like(dk) if dk.is_contiguous() else _new_like(k)
    else:
        _check_tensor("dv", dv, device, dtype, kshape)
    _set_array(p, "dout", dout), _set_array(p, "out", out)
    _set_array(p, "dq", dq), _set_array(p, "dk", dk), _set_array(p, "dv", dv)
    ref = ct.byref(p)
    keep = _workspace(p, workspace, _lib.gbmw_attention_workspace(ref, 1), device)
    _check(_lib.gbmw_attention_backward(ref))
    return dq, dk, dv


def _row_stride(name: str, t) -> int:
    """Row stride of a tensor whose last axis is normed; the axes before it have to be one stride."""
    cols = t.shape[-1]
    if t.is_contiguous():
        return cols
    if t.stride(-1) != 1 and cols > 1:
        _refuse(f"{name}: the values of a row are not next to each other")
    axes = [(n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n > 1]
    if not axes or not t.numel():
        return cols
    for (n, s), (n1, s1) in zip(axes, axes[1:]):
        if s != n1 * s1:
            _refuse(f"{name}: its rows are not one stride apart")
    return axes[-1][1]


def _norm_problem(x, weight, bias):
    device = _device_of("x", x, _DTYPE)
    shape, dtype = x.shape, x.dtype
    if len(shape) < 1:
        _refuse("x has no axis")
    p, cols = gbmw_layer_norm_problem(), shape[-1]
    _check_counts("x", cols)
    p.dtype = p.wdtype = _DTYPE[dtype]
    p.rows, p.cols, p.x_stride = x.numel() // max(1, cols), cols, _row_stride("x", x)
    p.x, p.stream = x.data_ptr(), _raw_stream(device)
    if weight is not None or bias is not None:
        wdtype = getattr(bias if weight is None else weight, "dtype", None)
        p.wdtype = _DTYPE.get(wdtype, -1)
        if weight is not None:
            p.weight = _column("weight", weight, device, wdtype, cols)
        if bias is not None:
            p.bias = _column("bias", bias, device, wdtype, cols)
    return p, device


def _column(name: str, t, device: int, dtype, cols: int) -> int:
    _check_tensor(name, t, device, dtype, (cols,))
    if not t.is_contiguous():
        _refuse(f"{name} is not contiguous")
    return t.data_ptr()


@_on_stream
def gbmw_layer_norm_workspace(x, weight=None) -> int:
    """Bytes of workspace of the backward call."""
    n = _lib.gbmw_layer_norm_workspace(ct.byref(_norm_problem(x, weight, None)[0]))
    if n < 0:
        raise GbmwError(GBMW_ERR_INVALID_ARG, gbmw_last_error())
    return n


@_on_stream
def gbmw_layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, y=None):
    """y like x, mean and rstd float32 of x's shape without its last axis.  x: float32, float16 or bfloat16 GPU
    tensor; weight, bias: of x's type or float32.  y: made here unless given (it may be x).  stream=: as everywhere.
    Not recorded by autograd: gradients come from gbmw_layer_norm_backward."""
    p, device = _norm_problem(x, weight, bias)
    if y is None:
        y, p.y_stride = _new_like(x), p.cols
    else:
        _check_tensor("y", y, device, x.dtype, x.shape)
        p.y_stride = _row_stride("y", y)
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device="cuda")
    rstd = torch.empty_like(mean)
    p.eps, p.y, p.mean, p.rstd = eps, y.data_ptr(), mean.data_ptr(), rstd.data_ptr()
    _check(_lib.gbmw_layer_norm_forward(ct.byref(p)))
    return y, mean, rstd


@_on_stream
def gbmw_layer_norm_backward(dy, x, weight, mean, rstd, bias: bool = True, dx=None, workspace=None):
    """dx, dweight, dbias from dy and the forward call's x, weight, mean and rstd.  weight None: no dweight; bias
    False: no dbias.  Both are of weight's type (x's without one).  stream=: as everywhere."""
    p, device = _norm_problem(x, weight, None)
    if dx is None:
        dx, p.dx_stride = _new_like(x), p.cols
    else:
        _check_tensor("dx", dx, device, x.dtype, x.shape)
        p.dx_stride = _row_stride("dx", dx)
    _check_tensor("dy", dy, device, x.dtype, x.shape)
    p.dy_stride = _row_stride("dy", dy)
    p.dx, p.dy = dx.data_ptr(), dy.data_ptr()
    for name, t in (("mean", mean), ("rstd", rstd)):
        _check_tensor(name, t, device, torch.float32, x.shape[:-1])
        if not t.is_contiguous():
            _refuse(f"{name} is not contiguous")
    p.mean, p.rstd = mean.data_ptr(), rstd.data_ptr()
    wdtype = x.dtype if weight is None else weight.dtype
    dweight = dbias = keep = None
    if weight is not None:
        dweight = torch.empty(p.cols, dtype=wdtype, device="cuda")
        p.dweight = dweight.data_ptr()
    if bias:
        dbias = torch.empty(p.cols, dtype=wdtype, device="cuda")
        p.dbias = dbias.data_ptr()
    ref = ct.byref(p)
    if weight is not None or bias:
        keep = _workspace(p, workspace, _lib.gbmw_layer_norm_workspace(ref), device)
    _check(_lib.gbmw_layer_norm_backward(ref))
    return dx, dweight, dbias


class GradientList:
    """Owns a gbmw_gradient_list and keeps its tensors; freed by gbmw_gradient_list_destroy or with this object."""

    def __init__(self):
        self.handle = ct.c_void_p(None)
        self._keep = ()

    def __del__(self):
        try:
            gbmw_gradient_list_destroy(self)
        except Exception:
            pass


def gbmw_gradient_list_create(grads, outs=None, norm_only: bool = False) -> GradientList:
    """A list of gradients (contiguous GPU tensors) and of the tensors that their clipped values go to, of the same
    types or float32; by default the gradients themselves.  norm_only: the list is for the norm alone, and
    gbmw_clip_gradients writes no tensor.  The tensors have to stay where they are."""
    grads = list(grads)
    if norm_only and outs is not None:
        _refuse("outputs of a list for the norm alone")
    outs = grads if outs is None else list(outs)
    if len(outs) != len(grads):
        _refuse(f"{len(grads)} gradients, {len(outs)} outputs")
    for i, (g, o) in enumerate(zip(grads, outs)):
        _device_of(f"gradient {i}", g, _DTYPE), _device_of(f"output {i}", o, _DTYPE)
        if o.numel() != g.numel() or not g.is_contiguous() or not o.is_contiguous():
            _refuse(f"tensor {i}: sizes {g.numel()} and {o.numel()}, or not contiguous")
    n = len(grads)
    pointers = lambda ts: (ct.c_void_p * max(1, n))(*[t.data_ptr() or None for t in ts])
    types = lambda ts: (ct.c_int32 * max(1, n))(*[_DTYPE.get(t.dtype, -1) for t in ts])
    numel = (ct.c_int64 * max(1, n))(*[g.numel() for g in grads])
    lst = GradientList()
    _check(_lib.gbmw_gradient_list_create(n, pointers(grads), None if norm_only else pointers(outs), numel, types(grads),
                                          None if norm_only else types(outs), ct.byref(lst.handle)))
    lst._keep = (grads, outs)
    return lst


@_on_stream
def gbmw_clip_gradients(lst: GradientList, max_norm: float, scale: float = 1.0, norm=None):
    """Writes the list's outputs, if it has any; returns the norm before clipping, a float32 GPU tensor [1] (norm, if given).
    stream=: as everywhere."""
    if norm is None:
        norm = torch.empty(1, dtype=torch.float32, device="cuda")
    elif _device_of("norm", norm, (torch.float32,)) < 0 or norm.numel() < 1:
        _refuse("norm is empty")
    _check(_lib.gbmw_clip_gradients(lst.handle, max_norm, scale, norm.data_ptr(), _raw_stream(norm.get_device())))
    return norm


def gbmw_gradient_list_destroy(lst: GradientList) -> None:
    if lst.handle:
        _lib.gbmw_gradient_list_destroy(lst.handle)
        lst.handle = ct.c_void_p(None)
        lst._keep = ()


RmsNorm = collections.namedtuple("RmsNorm", "y h rstd q scale")
_QTYPE = {torch.float8_e4m3fn: GBMW_E4M3, torch.int8: GBMW_I8}


def _rms_problem(x, weight):
    device = _device_of("x", x, _DTYPE)
    shape, dtype = x.shape, x.dtype
    if len(shape) < 1:
        _refuse("x has no axis")
    p, cols = gbmw_rms_norm_problem(), shape[-1]
    _check_counts("x", cols)
    p.dtype = p.wdtype = _DTYPE[dtype]
    p.rows, p.cols, p.x_stride = x.numel() // max(1, cols), cols, _row_stride("x", x)
    p.x, p.stream = x.data_ptr(), _raw_stream(device)
    if weight is not None:
        wdtype = getattr(weight, "dtype", None)
        p.wdtype = _DTYPE.get(wdtype, -1)
        p.weight = _column("weight", weight, device, wdtype, cols)
    return p, device


def _rows(name: str, t, device: int, dtype, shape) -> tuple:
    """Where t's rows are, and how far apart."""
    _check_tensor(name, t, device, dtype, shape)
    return t.data_ptr(), _row_stride(name, t)


@_on_stream
def gbmw_rms_norm_workspace(x, weight=None) -> int:
    """Bytes of workspace of the backward call (0 for a few rows)."""
    n = _lib.gbmw_rms_norm_workspace(ct.byref(_rms_problem(x, weight)[0]))
    if n < 0:
        raise GbmwError(GBMW_ERR_INVALID_ARG, gbmw_last_error())
    return n


@_on_stream
def gbmw_rms_norm_forward(x, weight=None, eps: float = 1e-5, residual=None, qtype=None, group: int = 0,
                          want_y: bool = True, y=None, h=None, q=None):
    """RmsNorm(y, h, rstd, q, scale) of x, a float32, float16 or bfloat16 GPU tensor whose last axis is normed, after
    the addition of residual, if there is one.  weight: of x's type or float32.  y: like x, None unless want_y.
    h: x + residual; without a residual x itself, or None where y is written over it (no backward call can follow).
    rstd: float32 of x's shape without its last axis.  qtype (torch.float8_e4m3fn or torch.int8): q holds y in 8 bits, with
    scale (float32, of x's shape but for the last axis) for each row, or for each `group` (32, 64 or 128) columns; None
    without a qtype.  y, h, q: made here unless given (y or h may be x or residual).  stream=: as everywhere.  Not recorded by autograd: gradients come from
    gbmw_rms_norm_backward."""
    p, device = _rms_problem(x, weight)
    shape, dtype = x.shape, x.dtype
    p.eps = eps
    if y is not None:
        p.y, p.y_stride = _rows("y", y, device, dtype, shape)
    elif want_y:
        y = _new_like(x)
        p.y, p.y_stride = y.data_ptr(), p.cols
    if residual is not None:
        p.residual, p.residual_stride = _rows("residual", residual, device, dtype, shape)
        if h is None:
            h = _new_like(x)
            p.h, p.h_stride = h.data_ptr(), p.cols
        else:
            p.h, p.h_stride = _rows("h", h, device, dtype, shape)
    elif h is not None:
        _refuse("h without a residual is x")
    elif y is None or y.data_ptr() != x.data_ptr() or not p.rows:
        h = x
    scale = None
    if qtype is not None:
        p.qtype, p.group = _QTYPE.get(qtype, -1), group
        if q is None:
            q = _new_like(x, qtype)
            p.q, p.q_stride = q.data_ptr(), p.cols
        else:
            p.q, p.q_stride = _rows("q", q, device, qtype, shape)
        scale = x.new_empty((*shape[:-1], -(-p.cols // group) if group > 0 else 1), dtype=torch.float32)
        p.scale = scale.data_ptr()
    elif q is not None:
        _refuse("q without a qtype")
    rstd = torch.empty(shape[0] if len(shape) == 2 else shape[:-1], dtype=torch.float32, device="cuda")   # a number is faster
    p.rstd = rstd.data_ptr()
    _check(_lib.gbmw_rms_norm_forward(ct.byref(p)))
    return RmsNorm(y, h, rstd, q, scale)


@_on_stream
def gbmw_rms_norm_backward(dy, h, weight, rstd, dres=None, dx=None, workspace=None):
    """dx (of x and of the residual) and dweight from dy and the forward call's h, weight and rstd.  dres: the gradient
    that reaches h past the norm, added to dx.  weight None: no dweight.  dx: made here unless given (it may be dy or
    dres).  stream=: as everywhere."""
    p, device = _rms_problem(h, weight)
    shape, dtype = h.shape, h.dtype
    p.dy, p.dy_stride = _rows("dy", dy, device, dtype, shape)
    if dres is not None:
        p.dres, p.dres_stride = _rows("dres", dres, device, dtype, shape)
    if dx is None:
        dx = _new_like(h)
        p.dx, p.dx_stride = dx.data_ptr(), p.cols
    else:
        p.dx, p.dx_stride = _rows("dx", dx, device, dtype, shape)
    _check_tensor("rstd", rstd, device, torch.float32, shape[:-1])
    if not rstd.is_contiguous():
        _refuse("rstd is not contiguous")
    p.rstd = rstd.data_ptr()
    ref, dweight, keep = ct.byref(p), None, None
    if weight is not None:
        dweight = torch.empty_like(weight)
        p.dweight = dweight.data_ptr()
        need = _lib.gbmw_rms_norm_workspace(ref)
        keep = _workspace(p, workspace, need, device) if need else None
    _check(_lib.gbmw_rms_norm_backward(ref))
    return dx, dweight


_SCALING = dict(none=GBMW_ROTARY_NONE, linear=GBMW_ROTARY_LINEAR, base=GBMW_ROTARY_BASE, ramp=GBMW_ROTARY_RAMP)


@_on_stream
def gbmw_rotary_frequencies(rot: int, theta: float = 10000.0, scaling: str = "none", by: float = 1.0,
                            original: float = 0.0, slow: float = 1.0, fast: float = 32.0):
    """Radians per position of rot / 2 pairs, a float64 GPU tensor.  scaling: "none", "linear", "base" or "ramp", for
    contexts `by` times as long as those that theta is made for (of `original` positions, with "ramp")."""
    _check_counts("rot", abs(rot))
    if scaling not in _SCALING:
        _refuse(f"scaling {scaling!r} is none of {', '.join(_SCALING)}")
    freq = np.empty(max(0, rot // 2))
    _check(_lib.gbmw_rotary_frequencies(rot, theta, _SCALING[scaling], by, original, slow, fast, freq.ctypes.data))
    return torch.from_numpy(freq).to("cuda")


def _rotary(call, q, k, freq, positions, len_x, interleaved, factor, q_out, k_out):
    device = _device_of("q", q, _DTYPE)
    shape, dtype = q.shape, q.dtype
    if len(shape) != 4:
        _refuse(f"q has {q.dim()} dimensions, not [B][L][Hq][D]")
    B, L, Hq, D = shape
    Hk = 0
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            _refuse("k is not a tensor [B][L][Hk][D]")
        Hk = k.shape[2]
        _check_tensor("k", k, device, dtype, (B, L, Hk, D))
    elif k_out is not None:
        _refuse("k_out without k")
    _check_counts("q and k", B | L | Hq | Hk | D)
    if not isinstance(freq, torch.Tensor) or freq.dim() != 1:
        _refuse("freq is not a tensor [rot / 2]")
    _check_tensor("freq", freq, device, torch.float64, freq.shape)
    if not freq.is_contiguous():
        _refuse("freq is not contiguous")
    position = position_stride = length = k_at = k_to = 0
    k_strides = k_to_strides = (0, 0, 0)
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
            _refuse("positions is not a tensor [B][L]")
        _check_tensor("positions", positions, device, torch.int32, (B, L))
        position_stride, step = positions.stride()
        if L > 1 and step != 1:
            _refuse("positions of one sample are not next to each other")
        position = positions.data_ptr()
    if len_x is not None:
        length = _length("len_x", len_x, device, B)
    if q_out is None:
        q_out = _new_like(q)
    else:
        _check_tensor("q_out", q_out, device, dtype, shape)
    if k is not None:
        if k_out is None:
            k_out = _new_like(k)
        else:
            _check_tensor("k_out", k_out, device, dtype, k.shape)
        k_at, k_to, k_strides, k_to_strides = k.data_ptr(), k_out.data_ptr(), _strides("k", k), _strides("k_out", k_out)
    if not -3.4e38 < factor < 3.4e38:
        _refuse(f"factor={factor}")     # what does not pack as 32 bits
    p = gbmw_rotary_problem.from_buffer_copy(_ROTARY.pack(
        _DTYPE[dtype], B, L, Hq, Hk, D, 2 * min(freq.shape[0], 1 << 20), 1 if interleaved else 0, factor, freq.data_ptr(), position,
        position_stride, length, q.data_ptr(), k_at, *_strides("q", q), *k_strides, q_out.data_ptr(), k_to,
        *_strides("q_out", q_out), *k_to_strides, _raw_stream(device)))
    _check(call(ct.byref(p)))
    return q_out, k_out


@_on_stream
def gbmw_rotary_forward(q, k, freq, positions=None, len_x=None, interleaved: bool = False, factor: float = 1.0,
                        q_out=None, k_out=None):
    """q [B][L][Hq][D] and k [B][L][Hk][D] (or None) with the first 2 * len(freq) values of each head turned by their
    rows' positions: float32, float16 or bfloat16 GPU tensors with any strides whose last one is 1.  freq: float64,
    radians per position (gbmw_rotary_frequencies).  positions: int32 [B][L]; by default a row's number.  len_x: int32
    [B]; rows from there on are left as they were (in outputs made here: as memory was).  q_out, k_out: made here unless
    given (they may be q and k).
    stream=: as everywhere.  Not recorded by autograd: gradients come from gbmw_rotary_backward."""
    return _rotary(_lib.gbmw_rotary_forward, q, k, freq, positions, len_x, interleaved, factor, q_out, k_out)


@_on_stream
def gbmw_rotary_backward(dq, dk, freq, positions=None, len_x=None, interleaved: bool = False, factor: float = 1.0,
                         q_out=None, k_out=None):
    """The gradients of the forward call's q and k from those of its results, dq and dk (or None), by the same freq,
    positions, len_x, interleaved and factor.  q_out, k_out: made here unless given (they may be dq and dk)."""
    return _rotary(_lib.gbmw_rotary_backward, dq, dk, freq, positions, len_x, interleaved, factor, q_out, k_out)


class AdamWList:
    """Owns a gbmw_adamw_list and keeps its tensors; freed by gbmw_adamw_list_destroy or with this object."""

    def __init__(self):
        self.handle = ct.c_void_p(None)
        self._keep = ()

    def __del__(self):
        try:
            gbmw_adamw_list_destroy(self)
        except Exception:
            pass


def gbmw_adamw_list_create(params, grads, m, v, m_scales=None, v_scales=None, copies=None, weight_decay=0.0) -> AdamWList:
    """A list of parameters (contiguous GPU tensors of float32, float16 or bfloat16), their gradients, and their states:
    m and v in float32, or in float8_e4m3fn (v: of the second moment's square root), then with m_scales and v_scales in
    float32, one for each 256 elements.  copies: tensors of 16 bits that get the new parameters too (None, or None in
    the place of one).  weight_decay: a number, or one for each tensor.  The tensors have to stay where they are."""
    params, grads, m, v = list(params), list(grads), list(m), list(v)
    n = len(params)
    wide = torch.float8_e4m3fn if m and getattr(m[0], "dtype", None) == torch.float8_e4m3fn else torch.float32
    bits = 8 if wide == torch.float8_e4m3fn else 32
    scales = [list(s) if s is not None else [None] * n for s in (m_scales, v_scales)]
    copies = [None] * n if copies is None else list(copies)
    decay = list(weight_decay) if isinstance(weight_decay, collections.abc.Iterable) and not hasattr(weight_decay, "__float__") \
        else [weight_decay] * n
    for name, ts in (("gradients", grads), ("m", m), ("v", v), ("m_scales", scales[0]), ("v_scales", scales[1]),
                     ("copies", copies), ("weight_decay", decay)):
        if len(ts) != n:
            _refuse(f"{n} parameters, {len(ts)} {name}")
    if bits == 32 and n and not (m_scales is None and v_scales is None):
        _refuse("states of 32 bits have no scales")
    tensors = (gbmw_adamw_tensor * max(1, n))()
    for i, t in enumerate(tensors[:n]):
        device = _device_of(f"parameter {i}", params[i], _DTYPE)
        shape = params[i].shape
        _device_of(f"gradient {i}", grads[i], _DTYPE)
        arrays = [("param", params[i], params[i].dtype, shape), ("grad", grads[i], grads[i].dtype, shape),
                  ("m", m[i], wide, shape), ("v", v[i], wide, shape)]
        if bits == 8:
            blocks = ((params[i].numel() + 255) // 256,)
            arrays += [("m_scale", scales[0][i], torch.float32, blocks), ("v_scale", scales[1][i], torch.float32, blocks)]
        if copies[i] is not None:
            arrays.append(("copy", copies[i], getattr(copies[i], "dtype", None), shape))
        for name, x, dtype, size in arrays:
            _check_tensor(f"{name} of tensor {i}", x, device, dtype, size)
            if not x.is_contiguous():
                _refuse(f"{name} of tensor {i} is not contiguous")
            setattr(t, name, x.data_ptr() or None)
        t.numel, t.grad_dtype, t.dtype = params[i].numel(), _DTYPE[grads[i].dtype], _DTYPE[params[i].dtype]
        t.copy_dtype, t.weight_decay = -1 if copies[i] is None else _DTYPE.get(copies[i].dtype, -1), decay[i]
    lst = AdamWList()
    _check(_lib.gbmw_adamw_list_create(n, tensors, bits, ct.byref(lst.handle)))
    lst._keep = (params, grads, m, v, scales, copies)
    return lst


def _scalar_now(name: str, t, dtype) -> int:
    _device_of(name, t, (dtype,))
    if t.numel() < 1:
        _refuse(f"{name} is empty")
    return t.data_ptr()


@_on_stream
def gbmw_adamw_step(lst: AdamWList, lr, step, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                    scale: float = 1.0, norm=None, max_norm: float = float("inf"), seed: int = 0) -> None:
    """One step of the list's parameters and states.  lr: a number, or a float32 GPU tensor that is read when the step
    runs; step: the step's number from 1 on, or an int64 GPU tensor.  scale: of the gradients, the inverse of a loss scale.
    norm: of the gradients times scale, what gbmw_clip_gradients returned for a list with norm_only and the same scale: the
    gradients are clipped to max_norm as they are read, and the step is left out where it is not finite.  seed (up to
    2^32 - 1): of the rounding of states of 8 bits.  A training with such states gives one other than 0: 0 rounds to the
    nearest, which leaves moments that move by less than half a step at a time (second moments, by a thousandth of
    themselves) where they are.  stream=: as everywhere."""
    if not 0 <= seed < 1 << 32:
        _refuse(f"seed={seed} is not in 0..2^32 - 1")       # its lower bits alone may be 0, which rounds to the nearest
    o = gbmw_adamw_options(0.0, beta1, beta2, eps, scale, max_norm, 1, seed)
    if isinstance(lr, torch.Tensor):
        o.lr_now = _scalar_now("lr", lr, torch.float32)
    else:
        o.lr = lr
    if isinstance(step, torch.Tensor):
        o.step_now = _scalar_now("step", step, torch.int64)
    else:
        o.step = step
    if norm is not None:
        o.norm = _scalar_now("norm", norm, torch.float32)
    _check(_lib.gbmw_adamw_step(lst.handle, ct.byref(o), _raw_stream(_current_device())))


def gbmw_adamw_list_destroy(lst: AdamWList) -> None:
    if lst.handle:
        _lib.gbmw_adamw_list_destroy(lst.handle)
        lst.handle = ct.c_void_p(None)
        lst._keep = ()


def gbmw_export_tables(ctx: Context, instance: int, l0: int = 0, l1: int | None = None,
                       want_C: bool = True, want_A: bool = True):
    """C [l1-l0][E+1][S] float32 and A [l1-l0][E+1][S] uint8 (None if not wanted)."""
    if l1 is None:
        l1 = int(ctx.L[instance])
    n = max(0, l1 - l0)
    C = np.empty((n, ctx.E + 1, ctx.S), np.float32) if want_C else None
    A = np.empty((n, ctx.E + 1, ctx.S), np.uint8) if want_A else None
    _check(_lib.gbmw_export_tables(ctx.handle, instance, l0, l1,
                                   C.ctypes.data if want_C else None,
                                   A.ctypes.data if want_A else None))
    return C, A


def gbmw_last_solve_ms(ctx: Context):
    """(total_ms, minplus_ms, minplus_launches) of the last solve."""
    a, b, n = ct.c_float(), ct.c_float(), ct.c_int32()
    _check(_lib.gbmw_last_solve_ms(ctx.handle, ct.byref(a), ct.byref(b), ct.byref(n)))
    return a.value, b.value, n.value


def gbmw_last_solve_work(ctx: Context, launch: int = -1):
    """(units of 256 budgets that read one column, other groups of 64 that do, candidate updates that the
    bounds leave, rows of the groups that read several columns) of the last counted solve: of one min-plus
    launch, or summed over all (launch = -1)."""
    w = (ct.c_uint64 * 4)()
    _check(_lib.gbmw_last_solve_work(ctx.handle, launch, w))
    return tuple(int(x) for x in w)


def gbmw_destroy(ctx: Context) -> None:
    if ctx.handle:
        _lib.gbmw_destroy(ctx.handle)
        ctx.handle = ct.c_void_p(None)
        ctx._keep = ()

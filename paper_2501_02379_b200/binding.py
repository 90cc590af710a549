"""Thin ctypes binding of the C ABI in include/tgrad.h.

Argument marshalling only: every step of the optimizer runs in the CUDA
library.  PyTorch is used to own device memory and streams.  If the library
is missing, loading raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import weakref
from typing import List, NamedTuple, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtgrad.so")
MAX_NDIM = 8
NUM_STAGES = 5
STAGE_NAMES = ["proj_tail", "proj_chain", "mode1_adam", "back_chain", "back_tail"]

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_BUFFER_TOO_SMALL, ERR_CUDA, ERR_NO_CONVERGE, ERR_NONFINITE, ERR_BAD_STATE = range(8)
ERR_TOO_LARGE = 8
NOALLOC_MAX_NUMEL = 1 << 26
FLAG_NO_CONVERGE, FLAG_NONFINITE, FLAG_COPY_TIMEOUT = 1, 2, 4
C64, C32H, C32B, R32, R16H, R16B = range(6)
COMPOSITIONS = {"us_lr": 0, "lr_us": 1, "sum": 2}
STRATEGIES = {"topk": 0, "randk": 1, "probk": 2}
WHAT_OMEGA, WHAT_M_L, WHAT_V_L, WHAT_M_S, WHAT_V_S, WHAT_CORE, WHAT_N_L, WHAT_N_S = 1, 2, 3, 4, 5, 6, 7, 8
WHAT_GRAM_BASE, WHAT_FACTOR_BASE = 32, 64


class TgradConfig(C.Structure):
    _fields_ = [
        ("ndim", C.c_int32),
        ("dims", C.c_int64 * MAX_NDIM),
        ("ranks", C.c_int32 * MAX_NDIM),
        ("k", C.c_int64),
        ("T", C.c_int32),
        ("lr", C.c_float), ("alpha", C.c_float), ("lambda_", C.c_float),
        ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
        ("weight_decay", C.c_float),
        ("wg_dtype", C.c_int32),
        ("auto_refresh", C.c_int32),
        ("jacobi_max_sweeps", C.c_int32),
        ("jacobi_tol", C.c_float),
        ("warm_refresh", C.c_int32),
        ("hooi_iters", C.c_int32),
        ("composition", C.c_int32),
        ("sparse_strategy", C.c_int32),
        ("seed", C.c_uint64),
    ]


class TgradTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("numel", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class TgradAdamwTensor(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("grad", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
                ("master", C.c_void_p), ("numel", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class TgradAdamwConfig(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("step", C.c_int64), ("grad_scale", C.c_void_p)]


class TgradLogits(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("rows", C.c_int64), ("vocab", C.c_int64), ("row_stride", C.c_int64),
                ("targets", C.c_void_p), ("dtype", C.c_int32), ("temperature", C.c_double)]


class TgradPolicyArgs(C.Structure):
    _fields_ = [("old_logp", C.c_void_p), ("ref_logp", C.c_void_p), ("advantages", C.c_void_p), ("weights", C.c_void_p),
                ("clip_low", C.c_float), ("clip_high", C.c_float), ("kl_coef", C.c_float), ("entropy_coef", C.c_float),
                ("grad_scale", C.c_float), ("reserved", C.c_float), ("stats", C.c_void_p), ("logp", C.c_void_p),
                ("entropy", C.c_void_p), ("dlogits", C.c_void_p), ("dlogits_stride", C.c_int64)]


class TgradPreferenceArgs(C.Structure):
    _fields_ = [("starts", C.c_void_p), ("ref_logp", C.c_void_p), ("pairs", C.c_int32), ("beta", C.c_float),
                ("label_smoothing", C.c_float), ("grad_scale", C.c_float), ("loss", C.c_void_p), ("rewards", C.c_void_p),
                ("logp", C.c_void_p), ("dlogits", C.c_void_p), ("dlogits_stride", C.c_int64)]


class TgradError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None

EXPORTS = [
    "tgrad_state_bytes", "tgrad_init_state", "tgrad_step", "tgrad_refresh_subspace", "tgrad_step_batched",
    "tgrad_refresh_subspace_batched", "tgrad_query_status", "tgrad_export_state", "tgrad_import_state",
    "tgrad_set_step", "tgrad_destroy_state", "tgrad_status_string", "tgrad_launch_count",
    "tgrad_set_stage_timing", "tgrad_get_stage_times", "tgrad_select_topk_noalloc", "tgrad_diagnostics",
    "tgrad_step_scaled", "tgrad_step_batched_scaled", "tgrad_grad_norm_bytes", "tgrad_grad_norm", "tgrad_clip_grads",
    "tgrad_adamw_step", "tgrad_token_logprob", "tgrad_token_logprob_backward", "tgrad_policy_loss_bytes",
    "tgrad_policy_loss", "tgrad_preference_loss_bytes", "tgrad_preference_loss", "tgrad_set_copy_limit",
    "tgrad_packed_bytes", "tgrad_act_pack", "tgrad_act_unpack", "tgrad_gated_act", "tgrad_gated_act_backward",
    "tgrad_residual_norm", "tgrad_residual_norm_backward_bytes", "tgrad_residual_norm_backward", "tgrad_weight_grad_bytes",
    "tgrad_weight_grad",
]


def lib() -> C.CDLL:
    """Load libtgrad.so (once).  Raises OSError if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: build it with paper_2501_02379_b200.build.build() "
                          "(there is no CPU fallback)")
        l = C.CDLL(LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        cfgp = C.POINTER(TgradConfig)
        l.tgrad_state_bytes.argtypes = [cfgp, C.POINTER(sz), C.POINTER(sz)]
        l.tgrad_init_state.argtypes = [cfgp, vp, sz, vp, sz, vp, C.POINTER(vp)]
        l.tgrad_step.argtypes = [vp, vp, vp, vp]
        l.tgrad_refresh_subspace.argtypes = [vp, vp, vp]
        l.tgrad_step_batched.argtypes = [C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.c_int32, vp]
        l.tgrad_refresh_subspace_batched.argtypes = [C.POINTER(vp), C.POINTER(vp), C.c_int32, vp]
        l.tgrad_query_status.argtypes = [vp, vp, C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
        l.tgrad_export_state.argtypes = [vp, C.c_int32, vp, sz, vp]
        l.tgrad_import_state.argtypes = [vp, C.c_int32, vp, sz, vp]
        l.tgrad_set_step.argtypes = [vp, C.c_int64]
        l.tgrad_destroy_state.argtypes = [vp]
        l.tgrad_status_string.argtypes = [C.c_int]
        l.tgrad_status_string.restype = C.c_char_p
        l.tgrad_launch_count.argtypes = []
        l.tgrad_launch_count.restype = C.c_int64
        l.tgrad_set_stage_timing.argtypes = [vp, C.c_int32]
        l.tgrad_get_stage_times.argtypes = [vp, vp, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
        l.tgrad_select_topk_noalloc.argtypes = [vp, C.c_int64, C.c_int64, C.c_int32, vp, vp, vp]
        l.tgrad_diagnostics.argtypes = [vp, vp, vp, C.POINTER(C.c_double)]
        l.tgrad_step_scaled.argtypes = [vp, vp, vp, vp, vp]
        l.tgrad_step_batched_scaled.argtypes = [C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.c_int32, vp, vp]
        l.tgrad_grad_norm_bytes.argtypes = [C.c_int32, C.POINTER(sz)]
        l.tgrad_grad_norm.argtypes = [vp, C.c_int32, C.c_float, vp, vp, sz, vp]
        l.tgrad_clip_grads.argtypes = [vp, C.c_int32, C.c_float, vp, vp, sz, vp]
        l.tgrad_adamw_step.argtypes = [vp, C.c_int32, vp, vp]
        l.tgrad_token_logprob.argtypes = [vp, vp, vp, vp, vp]
        l.tgrad_token_logprob_backward.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int64, vp]
        l.tgrad_policy_loss_bytes.argtypes = [C.c_int64, C.POINTER(sz)]
        l.tgrad_policy_loss.argtypes = [vp, vp, vp, sz, vp]
        l.tgrad_preference_loss_bytes.argtypes = [C.c_int64, C.c_int32, C.POINTER(sz)]
        l.tgrad_preference_loss.argtypes = [vp, vp, vp, sz, vp]
        l.tgrad_set_copy_limit.argtypes = [C.c_int32]
        l.tgrad_packed_bytes.argtypes = [C.c_int64, C.c_int64, C.POINTER(sz)]
        l.tgrad_act_pack.argtypes = [vp, C.c_int64, C.c_int64, C.c_int32, vp, vp]
        l.tgrad_act_unpack.argtypes = [vp, C.c_int64, C.c_int64, C.c_int32, vp, vp]
        l.tgrad_gated_act.argtypes = [vp, vp]
        l.tgrad_gated_act_backward.argtypes = [vp, vp]
        l.tgrad_residual_norm.argtypes = [vp, vp, vp]
        l.tgrad_residual_norm_backward_bytes.argtypes = [vp, C.POINTER(sz)]
        l.tgrad_residual_norm_backward.argtypes = [vp, vp, vp, sz, vp]
        l.tgrad_weight_grad_bytes.argtypes = [vp, C.POINTER(sz)]
        l.tgrad_weight_grad.argtypes = [vp, vp, sz, vp]
        for name in EXPORTS:
            if name not in ("tgrad_status_string", "tgrad_launch_count"):
                getattr(l, name).restype = C.c_int
        _lib = l
    return _lib


def status_string(s: int) -> str:
    return lib().tgrad_status_string(int(s)).decode()


def launch_count() -> int:
    return int(lib().tgrad_launch_count())


def _check(s: int, where: str) -> None:
    if s != OK:
        raise TgradError(s, where)


def make_config(shape: Sequence[int], ranks: Sequence[int], k: int, T: int, lr: float = 1e-3, alpha: float = 1.0,
                lam: float = 1.0, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                weight_decay: float = 0.0, half_storage: bool = False, bf16_storage: bool = False, auto_refresh: bool = True,
                jacobi_max_sweeps: int = 0, jacobi_tol: float = 0.0, warm_refresh: bool = False,
                hooi_iters: int = 0, composition: str = "us_lr", strategy: str = "topk", seed: int = 0) -> TgradConfig:
    if len(shape) > MAX_NDIM or len(shape) != len(ranks):
        raise ValueError("bad shape / ranks")
    cfg = TgradConfig()
    cfg.ndim = len(shape)
    for i, (d, r) in enumerate(zip(shape, ranks)):
        cfg.dims[i] = int(d)
        cfg.ranks[i] = int(r)
    cfg.k = int(k)
    cfg.T = int(T)
    cfg.lr, cfg.alpha, cfg.lambda_ = lr, alpha, lam
    cfg.beta1, cfg.beta2, cfg.eps = beta1, beta2, eps
    cfg.weight_decay = weight_decay
    cfg.wg_dtype = C32B if bf16_storage else (C32H if half_storage else C64)
    cfg.auto_refresh = 1 if auto_refresh else 0
    cfg.jacobi_max_sweeps = jacobi_max_sweeps
    cfg.jacobi_tol = jacobi_tol
    cfg.warm_refresh = 1 if warm_refresh else 0
    cfg.hooi_iters = int(hooi_iters)
    cfg.composition = COMPOSITIONS[composition]
    cfg.sparse_strategy = STRATEGIES[strategy]
    cfg.seed = int(seed)
    return cfg


def state_bytes(cfg: TgradConfig):
    p, w = C.c_size_t(0), C.c_size_t(0)
    _check(lib().tgrad_state_bytes(C.byref(cfg), C.byref(p), C.byref(w)), "tgrad_state_bytes")
    return int(p.value), int(w.value)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream
    return int(stream)


def _scalar_ptr(scale, index) -> Optional[int]:
    if scale is None:
        return None
    if scale.dtype is not _torch()[2] or scale.numel() != 1 or not scale.is_cuda or scale.get_device() != index:
        raise ValueError("a scale is an fp32 CUDA tensor of one entry on the gradients' device")
    return scale.data_ptr()


class TgradState:
    """One optimizer state (one weight tensor).  Device blocks are torch uint8
    tensors owned by this object; the library only borrows them."""

    def __init__(self, cfg: TgradConfig, device="cuda", stream=None):
        import torch
        self.cfg = cfg
        self.shape = tuple(int(cfg.dims[i]) for i in range(cfg.ndim))
        self.ranks = tuple(int(cfg.ranks[i]) for i in range(cfg.ndim))
        self.k = int(cfg.k)
        self.core_entries = int(np.prod(self.ranks, dtype=np.int64))
        pb, wb = state_bytes(cfg)
        self.persistent = torch.empty(max(pb, 256), dtype=torch.uint8, device=device)
        self.workspace = torch.empty(max(wb, 256), dtype=torch.uint8, device=device)
        h = C.c_void_p(0)
        _check(lib().tgrad_init_state(C.byref(cfg), self.persistent.data_ptr(), pb, self.workspace.data_ptr(), wb,
                                      _stream_ptr(stream), C.byref(h)), "tgrad_init_state")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().tgrad_destroy_state(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # --- the hot path -------------------------------------------------------------
    def step(self, weight, grad, stream=None):
        _check(lib().tgrad_step(self.handle, weight.data_ptr(), grad.data_ptr(), _stream_ptr(stream)), "tgrad_step")

    def step_scaled(self, weight, grad, scale, stream=None):
        """step() with the gradient multiplied by the device scalar `scale` (an fp32 tensor of one entry, such as the
        clipping coefficient grad_norm(...)[1:2]); costs no pass over the gradient."""
        _check(lib().tgrad_step_scaled(self.handle, weight.data_ptr(), grad.data_ptr(), _scalar_ptr(scale, grad.get_device()), _stream_ptr(stream)),
               "tgrad_step_scaled")
        if stream is not None and scale is not None:
            scale.record_stream(_as_stream(scale.get_device(), stream))

    def refresh_subspace(self, grad, stream=None):
        _check(lib().tgrad_refresh_subspace(self.handle, grad.data_ptr(), _stream_ptr(stream)),
               "tgrad_refresh_subspace")

    # --- status / inspection ---------------------------------------------------------
    def query_status(self, stream=None):
        flags, t = C.c_int32(0), C.c_int64(0)
        sweeps = (C.c_int32 * MAX_NDIM)()
        _check(lib().tgrad_query_status(self.handle, _stream_ptr(stream), C.byref(flags), C.byref(t), sweeps),
               "tgrad_query_status")
        return int(flags.value), int(t.value), [int(sweeps[i]) for i in range(self.cfg.ndim)]

    def _spec(self, what):
        k, p = self.k, self.core_entries
        if what == WHAT_OMEGA:
            return (k,), np.uint32
        if what in (WHAT_M_L, WHAT_CORE, WHAT_N_L):
            return self.ranks, np.complex64
        if what == WHAT_V_L:
            return self.ranks, np.float32
        if what in (WHAT_M_S, WHAT_N_S):
            return (k,), np.complex64
        if what == WHAT_V_S:
            return (k,), np.float32
        if WHAT_FACTOR_BASE <= what < WHAT_FACTOR_BASE + self.cfg.ndim:
            n = what - WHAT_FACTOR_BASE
            return (self.shape[n], self.ranks[n]), np.complex64
        if WHAT_GRAM_BASE <= what < WHAT_GRAM_BASE + self.cfg.ndim:
            n = what - WHAT_GRAM_BASE
            return (self.shape[n], self.shape[n]), np.complex64
        raise ValueError(what)

    def export(self, what, stream=None) -> np.ndarray:
        shape, dt = self._spec(what)
        out = np.empty(shape, dtype=dt)
        _check(lib().tgrad_export_state(self.handle, what, out.ctypes.data, out.nbytes, _stream_ptr(stream)),
               "tgrad_export_state")
        return out

    def import_(self, what, arr: np.ndarray, stream=None):
        shape, dt = self._spec(what)
        a = np.ascontiguousarray(arr, dtype=dt)
        if a.shape != tuple(shape):
            raise ValueError("shape mismatch")
        _check(lib().tgrad_import_state(self.handle, what, a.ctypes.data, a.nbytes, _stream_ptr(stream)),
               "tgrad_import_state")

    def factors(self) -> List[np.ndarray]:
        return [self.export(WHAT_FACTOR_BASE + n) for n in range(self.cfg.ndim)]

    def set_step(self, t: int):
        _check(lib().tgrad_set_step(self.handle, int(t)), "tgrad_set_step")

    def diagnostics(self, grad, stream=None):
        """(||G||_F, sparse share, low-rank reconstruction error relative to ||G||_F, orthonormality defect) of the last step."""
        out = (C.c_double * 4)()
        _check(lib().tgrad_diagnostics(self.handle, grad.data_ptr(), _stream_ptr(stream), out), "tgrad_diagnostics")
        return tuple(float(out[i]) for i in range(4))

    def set_stage_timing(self, on: bool):
        _check(lib().tgrad_set_stage_timing(self.handle, 1 if on else 0), "tgrad_set_stage_timing")

    def stage_times(self, stream=None):
        ms = (C.c_float * NUM_STAGES)()
        n = C.c_int32(0)
        _check(lib().tgrad_get_stage_times(self.handle, _stream_ptr(stream), ms, C.byref(n)), "tgrad_get_stage_times")
        return [float(ms[i]) for i in range(NUM_STAGES)], int(n.value)


def step_batched(states: Sequence[TgradState], weights, grads, stream=None, scale=None):
    """`scale`: device scalar that multiplies every gradient, as in TgradState.step_scaled."""
    n = len(states)
    hs = (C.c_void_p * n)(*[s.handle for s in states])
    ws = (C.c_void_p * n)(*[w.data_ptr() for w in weights])
    gs = (C.c_void_p * n)(*[g.data_ptr() for g in grads])
    if scale is not None:
        scale_p = _scalar_ptr(scale, grads[0].get_device() if n else scale.get_device())
        _check(lib().tgrad_step_batched_scaled(hs, ws, gs, n, scale_p, _stream_ptr(stream)), "tgrad_step_batched_scaled")
        if stream is not None:
            scale.record_stream(_as_stream(scale.get_device(), stream))
        return
    _check(lib().tgrad_step_batched(hs, ws, gs, n, _stream_ptr(stream)), "tgrad_step_batched")


def refresh_subspace_batched(states: Sequence[TgradState], grads, stream=None):
    n = len(states)
    hs = (C.c_void_p * n)(*[s.handle for s in states])
    gs = (C.c_void_p * n)(*[g.data_ptr() for g in grads])
    _check(lib().tgrad_refresh_subspace_batched(hs, gs, n, _stream_ptr(stream)), "tgrad_refresh_subspace_batched")


def select_topk_noalloc(grad, numel: int, k: int, omega_out, values_out, half_storage: bool = False, stream=None):
    """Top-k index set and values of `grad` through the entry point that allocates nothing:
    its scratch is a fixed array inside the library, so it serves callers that must not call
    cudaMalloc (allocator hooks, fully pre-partitioned device memory).  `omega_out` (k x uint32)
    and `values_out` (k x complex64 as float pairs) are device tensors the caller already owns.
    Calls share that scratch: keep them on one stream."""
    _check(lib().tgrad_select_topk_noalloc(grad.data_ptr(), int(numel), int(k), C32H if half_storage else C64,
                                           omega_out.data_ptr() if k else None, values_out.data_ptr() if k else None,
                                           _stream_ptr(stream)), "tgrad_select_topk_noalloc")


# --- around the step: gradient norm and clipping, AdamW, losses on logits ------------------------------------------
#
# Everything below runs on the current stream of the tensors' device, or on `stream` (a torch stream or its address).
# Results and workspaces that a call allocates belong to that stream.  As with torch's own operations the caller sees to
# the order of the streams: inputs have to be ready on the call's stream, and results are used on it or after it.

_torch_types = None       # torch, {dtype: tgrad_dtype}, torch.float32
_count_write = None       # tells autograd that tensors were written to


def _torch():
    global _torch_types, _count_write
    if _torch_types is None:
        import torch
        _count_write = torch.autograd.graph.increment_version
        _torch_types = (torch, {torch.float32: R32, torch.float16: R16H, torch.bfloat16: R16B, torch.complex64: C64}, torch.float32)
    return _torch_types


def _dtype_of(t) -> int:
    d = _torch()[1].get(t.dtype)
    if d is None:
        raise ValueError(f"unsupported dtype {t.dtype}")
    return d


def _dense(t) -> bool:
    """Every entry of the storage range belongs to the tensor once: contiguous in some order of the dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1):
        if stride != want:
            return False
        want *= size
    return True


def _same_places(a, b) -> bool:
    """Entries of the same index lie at the same place: equal shapes, and equal strides where a dimension has more than one
    entry."""
    return a.shape == b.shape and (a.stride() == b.stride() or a.numel() == 0 or
                                   all(s == t for s, t, n in zip(a.stride(), b.stride(), a.shape) if n > 1))


def _written(t) -> None:
    """autograd's check for operands that were overwritten is to see what a call has written to one of the caller's tensors."""
    if not t.is_inference():
        _count_write(t)


def _elsewhere(index, stream) -> bool:
    """Whether a call has to change the current device or stream first."""
    return stream is not None or index != _torch()[0]._C._cuda_getDevice()


def _as_stream(index, stream):
    if hasattr(stream, "cuda_stream"):
        return stream
    return _torch()[0].cuda.ExternalStream(int(stream), device=index)


def _there(index, stream, call, *args, **kw):
    """call(...) with the device `index` and the stream current.  The tensors among the arguments are marked as used on the
    stream, so that what the caller lets go of is not given to somebody else before the call has run."""
    torch = _torch()[0]
    with torch.cuda.device(index):
        if stream is None:
            return call(*args, **kw)
        stream = _as_stream(index, stream)
        if stream.device_index != index:
            raise ValueError("the stream belongs to another device than the tensors")
        with torch.cuda.stream(stream):
            result = call(*args, **kw)
        for x in args:
            for t in x.tensors if isinstance(x, TensorList) else x if isinstance(x, tuple) else (x,):
                if isinstance(t, torch.Tensor):
                    t.record_stream(stream)
        return result


def _raw_stream(index) -> int:
    return _torch()[0]._C._cuda_getCurrentRawStream(index)


# The argument structures as bytes (struct.pack costs a third of filling a ctypes structure).
_pack_logits = struct.Struct("@PqqqPid").pack
_pack_adamw = struct.Struct("@dddddqP").pack
_pack_policy = struct.Struct("@PPPPffffffPPPPq").pack
_pack_preference = struct.Struct("@PPifffPPPPq").pack
_workspace_bytes = {}


def _workspace(entry, *args) -> int:
    b = _workspace_bytes.get((entry, args))
    if b is None:
        n = C.c_size_t(0)
        _check(getattr(lib(), entry)(*args, C.byref(n)), entry)
        if len(_workspace_bytes) > 4096:
            _workspace_bytes.clear()
        b = _workspace_bytes[(entry, args)] = int(n.value)
    return b


class TensorList:
    """A list of CUDA tensors as the list calls take it, laid out once for tensors that stay where they are.  It keeps the
    tensors and the memory that they have when it is made, and the calls work on that memory: after anything that gives a
    tensor other memory, another shape or another type (module.to(), .half(), p.data = .., resize_(), a gradient that is a
    new tensor after zero_grad(set_to_none=True)) make a new list.  Every call that takes one also takes a plain sequence
    of tensors, which is laid out anew each time."""

    def __init__(self, tensors):
        self.tensors = tuple(tensors)
        for t in self.tensors:
            if not t.is_cuda or t.device != self.tensors[0].device:
                raise ValueError("the tensors of a list live on one CUDA device")
            if t.is_conj() or t.is_neg():
                raise ValueError("resolve lazy conjugations first")
            if not _dense(t):
                raise ValueError(f"a tensor of shape {tuple(t.shape)} and strides {t.stride()} is not dense in memory")
        n = len(self.tensors)
        self.array = (TgradTensor * max(n, 1))()
        for a, t in zip(self.array, self.tensors):
            a.data, a.numel, a.dtype = t.data_ptr(), t.numel(), _dtype_of(t)
        self.address = C.addressof(self.array)
        self._memory = [t.untyped_storage() for t in self.tensors]      # also after p.data = ..: nobody else is given it meanwhile
        self.floats = 64 + (2 + n + 63) // 64 * 64 + _workspace("tgrad_grad_norm_bytes", n) // 4      # results, then the workspace
        self._adamw = self._counters = None

    def written(self) -> None:
        """As _written, for all of the list: views count on what they are views of."""
        if self._counters is None:
            owners = [t if t._base is None else t._base for t in self.tensors]
            self._counters = tuple({id(t): t for t in owners if not t.is_inference()}.values())
        _count_write(self._counters)

    def __len__(self):
        return len(self.tensors)

    def device_index(self) -> int:
        return self.tensors[0].get_device() if self.tensors else _torch()[0].cuda.current_device()


def _as_list(x) -> TensorList:
    return x if isinstance(x, TensorList) else TensorList(x)


def _norm_call(name, grads, max_norm, stream):
    torch, _, f32 = _torch()
    grads = _as_list(grads)
    index = grads.device_index()
    if _elsewhere(index, stream):
        return _there(index, stream, _norm_call, name, grads, max_norm, None)
    n = len(grads.tensors)
    buf = torch.empty(grads.floats, dtype=f32, device=index)
    base, head = buf.data_ptr(), (2 + n + 63) // 64 * 64
    _check(getattr(lib(), name)(grads.address, n, max_norm, base, base + 4 * head, 4 * (grads.floats - head), _raw_stream(index)), name)
    if name == "tgrad_clip_grads":
        grads.written()
    return buf[:2 + n]


def grad_norm(grads, max_norm: float = float("inf"), stream=None):
    """Gradient norm over a list of tensors (fp32, fp16, bfloat16, complex64): an fp32 tensor [global norm, clipping
    coefficient min(1, max_norm / (norm + 1e-6)), norm of each tensor...] on the device.  Entry 1 as [1:2] is what
    step_scaled, step_batched and adamw_step take as a scale."""
    return _norm_call("tgrad_grad_norm", grads, max_norm, stream)


def clip_grads(grads, max_norm: float, stream=None):
    """grad_norm, and every gradient multiplied by the coefficient in place (autograd is told)."""
    return _norm_call("tgrad_clip_grads", grads, max_norm, stream)


def _adamw_array(params, grads, exp_avgs, exp_avg_sqs, masters):
    lists = [params, grads, exp_avgs, exp_avg_sqs] + ([masters] if masters is not None else [])
    if len({len(x) for x in lists}) != 1:
        raise ValueError("the lists differ in length")
    if any(x.device_index() != params.device_index() for x in lists):
        raise ValueError("the lists live on one device")
    # types, lengths and addresses are those that the lists keep (a tensor may have got other memory since), the order of the
    # entries is that of the tensors
    array = (TgradAdamwTensor * max(len(params), 1))()
    for i in range(len(params)):
        a, entries = array[i], [x.array[i] for x in lists]
        p, g, m, v = entries[:4]
        if g.dtype != p.dtype or v.dtype != R32 or m.dtype != (C64 if p.dtype == C64 else R32):
            raise ValueError("gradients have the weights' dtype, moments are fp32 (the first one complex64 for complex weights)")
        if masters is not None and (entries[4].dtype != R32 or p.dtype not in (R16H, R16B)):
            raise ValueError("master weights are the fp32 weights of 16-bit ones")
        for x, e in zip(lists[1:], entries[1:]):
            if e.numel != p.numel or not _same_places(x.tensors[i], params.tensors[i]):
                raise ValueError("weight, gradient and moments have the same shape and strides")
        a.weight, a.grad, a.exp_avg, a.exp_avg_sq = p.data, g.data, m.data, v.data
        a.master = entries[4].data if masters is not None else None
        a.numel, a.dtype = p.numel, p.dtype
    return array


def adamw_step(params, grads, exp_avgs, exp_avg_sqs, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
               eps: float = 1e-8, weight_decay: float = 0.0, grad_scale=None, masters=None, stream=None):
    """One AdamW step in place on a list of dense tensors (fp32, fp16, bfloat16 or complex64 weights; gradients of the
    same dtype; fp32 moments).  `step` counts from 1.  `grad_scale`: device scalar that multiplies the gradients.
    `masters`: fp32 weights of 16-bit ones, which are then what is updated.  For complex weights the second moment is
    real and takes the squared modulus.  autograd is told that the weights were written to.  TensorLists that are passed
    again in the same roles are laid out once; the first of them keeps that layout and none of the others, and nothing is
    kept of a call on plain sequences."""
    kept = getattr(params, "_adamw", None)      # (references to the other lists, None: no masters, and the layout)
    if kept is None or kept[0]() is not grads or kept[1]() is not exp_avgs or kept[2]() is not exp_avg_sqs or \
            (masters is not None if kept[3] is None else masters is None or kept[3]() is not masters):
        given = (params, grads, exp_avgs, exp_avg_sqs, masters)
        lists = [_as_list(x) if x is not None else None for x in given]
        array, params = _adamw_array(*lists), lists[0]
        if all(a is b for a, b in zip(given, lists)):
            params._adamw = tuple(None if x is None else weakref.ref(x) for x in lists[1:]) + (array,)
        grads, exp_avgs, exp_avg_sqs, masters = lists[1:]
    else:
        array = kept[4]
    index = params.device_index()
    if _elsewhere(index, stream):
        return _there(index, stream, adamw_step, params, grads, exp_avgs, exp_avg_sqs, step, lr, beta1, beta2, eps, weight_decay, grad_scale, masters)
    cfg = _pack_adamw(lr, beta1, beta2, eps, weight_decay, step, _scalar_ptr(grad_scale, index) or 0)
    _check(lib().tgrad_adamw_step(C.addressof(array), len(params.tensors), cfg, _raw_stream(index)), "tgrad_adamw_step")
    params.written()      # (no graph holds moments: they are not counted, 5 us a step for 40 tensors)
    if masters is not None:
        masters.written()


def _logits(logits, targets, temperature):
    """(the logits' description for the library, rows, vocabulary, device index); checks what the library cannot see."""
    torch, types, _ = _torch()
    if logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits are a CUDA tensor [rows, vocabulary]")
    rows, vocab = logits.shape
    d = types.get(logits.dtype)
    if d is None or d == C64:
        raise ValueError("logits are fp32, fp16 or bfloat16")
    stride, inner = logits.stride()
    if inner != 1 and vocab > 1:
        raise ValueError("the entries of a row of logits are adjacent")
    index = logits.get_device()
    if targets.dtype is not torch.int64 or targets.shape != (rows,) or targets.get_device() != index or not targets.is_contiguous():
        raise ValueError("targets are a contiguous int64 tensor [rows] on the logits' device")
    return _pack_logits(logits.data_ptr(), rows, vocab, stride if rows > 1 else vocab, targets.data_ptr(), d, temperature), rows, vocab, index


def _row_ptr(name, t, rows, index) -> int:
    """Address of an fp32 tensor [rows]."""
    if t.dtype is not _torch_types[2] or t.shape != (rows,) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous fp32 tensor [rows] on the logits' device")
    return t.data_ptr()


def _dlogits(logits, rows, vocab, out):
    """The gradient's tensor and row stride: `out` after a check, or a new one whose rows lie like those of the logits,
    so that both are accessed 16 bytes at a time."""
    if out is None:
        lead = (logits.data_ptr() & 15) // logits.element_size()
        stride = logits.stride(0) if rows > 1 else vocab
        if not vocab <= stride <= vocab + 128:
            stride = vocab
        if stride == vocab and not lead:
            return logits.new_empty((rows, vocab)), vocab
        return logits.new_empty(rows * stride + lead).as_strided((rows, vocab), (stride, 1), lead), stride
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device or (vocab > 1 and out.stride(1) != 1):
        raise ValueError("dlogits has the logits' shape, dtype and device, and the entries of a row are adjacent")
    return out, out.stride(0) if rows > 1 else vocab


def token_logprob(logits, targets, temperature: float = 1.0, stream=None):
    """(logp, lse, entropy), each fp32 [rows], of softmax(logits / temperature): log-probability of the row's target,
    log-sum-exp and entropy.  Rows with a negative target are ignored (0, and their logits are not read)."""
    desc, rows, _, index = _logits(logits, targets, temperature)
    if _elsewhere(index, stream):
        return _there(index, stream, token_logprob, logits, targets, temperature)
    torch, _, f32 = _torch_types
    out = torch.empty((3, rows), dtype=f32, device=index)
    base = out.data_ptr()
    _check(lib().tgrad_token_logprob(desc, base, base + 4 * rows, base + 8 * rows, _raw_stream(index)), "tgrad_token_logprob")
    return out.unbind(0)


def token_logprob_backward(logits, targets, lse, grad_logp, entropy=None, grad_entropy=None, temperature: float = 1.0, dlogits=None, stream=None):
    """Gradient of sum(grad_logp * logp + grad_entropy * entropy) with respect to the logits.  `dlogits` may be the
    logits themselves.  The probabilities are as exact as lse is in fp32: at low temperatures or for logits far from zero
    the losses' own gradients are more exact."""
    desc, rows, vocab, index = _logits(logits, targets, temperature)
    if _elsewhere(index, stream):
        return _there(index, stream, token_logprob_backward, logits, targets, lse, grad_logp, entropy, grad_entropy, temperature, dlogits)
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy needs the entropy of the forward call")
    lse_p, g_p = _row_ptr("lse", lse, rows, index), _row_ptr("grad_logp", grad_logp, rows, index)
    e_p = h_p = None
    if grad_entropy is not None:
        e_p, h_p = _row_ptr("entropy", entropy, rows, index), _row_ptr("grad_entropy", grad_entropy, rows, index)
    out, stride = _dlogits(logits, rows, vocab, dlogits)
    _check(lib().tgrad_token_logprob_backward(desc, lse_p, e_p, g_p, h_p, out.data_ptr(), stride, _raw_stream(index)),
           "tgrad_token_logprob_backward")
    if dlogits is not None:
        _written(dlogits)
    return out


def set_copy_limit(copies: int = -1) -> None:
    """For tests: the kernels that stream rows of logits through shared memory stop within the first row that takes more than so
    many copies (0: before any row, -1: never), those of a trained block after so many rows or steps.  The waits for further ones run
    out, which leaves NaN in the rows (tiles, sums) that were not finished.  For the whole process."""
    _check(lib().tgrad_set_copy_limit(int(copies)), "tgrad_set_copy_limit")


class PolicyLoss(NamedTuple):
    stats: "torch.Tensor"       # loss, and the weighted sums of the policy term, KL, entropy and clipped rows
    logp: "torch.Tensor"
    entropy: "torch.Tensor"
    dlogits: Optional["torch.Tensor"]


class PreferenceLoss(NamedTuple):
    loss: "torch.Tensor"        # scalar
    rewards: "torch.Tensor"     # beta * sum (logp - ref_logp) of each answer
    logp: "torch.Tensor"
    dlogits: Optional["torch.Tensor"]


def policy_loss(logits, targets, old_logp, advantages, weights, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, entropy_coef: float = 0.0, temperature: float = 1.0, grad_scale: float = 1.0,
                dlogits=None, forward_only: bool = False, stream=None) -> PolicyLoss:
    """Clipped policy loss with a KL term and an entropy bonus, and its gradient with respect to the logits in the same
    pass: loss = sum_i weights_i (-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(u) - u - 1)
    - entropy_coef H), r = exp(logp - old_logp), u = ref_logp - logp.  The weights carry mask and normalisation (what
    stands in or beside a row of weight 0 does not count); rows with a negative target are ignored, their logits too.  dlogits = grad_scale * d loss / d logits, ready for logits.backward(dlogits);
    `dlogits` may be the logits themselves."""
    desc, rows, vocab, index = _logits(logits, targets, temperature)
    if _elsewhere(index, stream):
        return _there(index, stream, policy_loss, logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl_coef,
                      entropy_coef, temperature, grad_scale, dlogits, forward_only)
    torch, _, f32 = _torch_types
    grad, stride = (None, 0) if forward_only else _dlogits(logits, rows, vocab, dlogits)
    ws = _workspace("tgrad_policy_loss_bytes", rows)
    out = torch.empty(ws // 4 + 5 + 2 * rows, dtype=f32, device=index)
    base = out.data_ptr()
    stats = base + ws
    args = _pack_policy(_row_ptr("old_logp", old_logp, rows, index), _row_ptr("ref_logp", ref_logp, rows, index) if ref_logp is not None else 0,
                        _row_ptr("advantages", advantages, rows, index), _row_ptr("weights", weights, rows, index), clip_low, clip_high,
                        kl_coef, entropy_coef, grad_scale, 0.0, stats, stats + 20, stats + 20 + 4 * rows,
                        grad.data_ptr() if grad is not None else 0, stride)
    _check(lib().tgrad_policy_loss(desc, args, base, ws, _raw_stream(index)), "tgrad_policy_loss")
    if dlogits is not None and grad is not None:
        _written(dlogits)
    _, stats, logp, entropy = out.split_with_sizes((ws // 4, 5, rows, rows))
    return PolicyLoss(stats, logp, entropy, grad)


def preference_loss(logits, targets, starts, ref_logp, beta: float = 0.1, label_smoothing: float = 0.0, temperature: float = 1.0,
                    grad_scale: float = 1.0, dlogits=None, forward_only: bool = False, stream=None) -> PreferenceLoss:
    """Loss on pairs of answers and its gradient with respect to the logits.  `starts`: int32 device tensor of
    2 * pairs + 1 row numbers, answers 2 b and 2 b + 1 are the chosen and the rejected one of pair b; rows of prompts
    have a negative target.  rewards_s = beta * sum (logp - ref_logp), h = rewards_chosen - rewards_rejected, loss = mean of
    -(1 - label_smoothing) log sigmoid(h) - label_smoothing log sigmoid(-h)."""
    desc, rows, vocab, index = _logits(logits, targets, temperature)
    if _elsewhere(index, stream):
        return _there(index, stream, preference_loss, logits, targets, starts, ref_logp, beta, label_smoothing, temperature, grad_scale, dlogits, forward_only)
    torch, _, f32 = _torch_types
    if starts.dtype is not torch.int32 or starts.dim() != 1 or starts.numel() % 2 != 1 or starts.get_device() != index or not starts.is_contiguous():
        raise ValueError("starts is a contiguous int32 tensor of 2 * pairs + 1 entries on the logits' device")
    pairs = starts.numel() // 2
    grad, stride = (None, 0) if forward_only else _dlogits(logits, rows, vocab, dlogits)
    ws = _workspace("tgrad_preference_loss_bytes", rows, pairs)
    out = torch.empty(ws // 4 + 1 + rows + 2 * pairs, dtype=f32, device=index)
    base = out.data_ptr()
    loss = base + ws
    args = _pack_preference(starts.data_ptr(), _row_ptr("ref_logp", ref_logp, rows, index), pairs, beta, label_smoothing, grad_scale, loss,
                            loss + 4 + 4 * rows, loss + 4, grad.data_ptr() if grad is not None else 0, stride)
    _check(lib().tgrad_preference_loss(desc, args, base, ws, _raw_stream(index)), "tgrad_preference_loss")
    if dlogits is not None and grad is not None:
        _written(dlogits)
    _, loss, logp, rewards = out.split_with_sizes((ws // 4, 1, rows, 2 * pairs))
    return PreferenceLoss(loss[0], rewards, logp, grad)


# --- a trained block: activations kept in 8 bits and what computes from them ---------------------------------------
#
# Matrices are [rows, width] CUDA tensors of fp32, fp16 or bfloat16 whose rows may lie apart (the entries of a row are
# adjacent); devices and streams as above.  Outputs must not overlap inputs.

class Packed(NamedTuple):
    """A matrix kept in 8.25 bits an entry (act_pack): blocks of 32 entries of a row share a power of two."""
    data: "torch.Tensor"        # uint8: the codes of all rows, then the blocks' exponents
    rows: int
    width: int
    dtype: "torch.dtype"        # what was packed, and what it is read back as


class GatedAct(NamedTuple):
    y: "torch.Tensor"
    a8: Optional[Packed]
    u8: Optional[Packed]


class GatedActGrads(NamedTuple):
    da: "torch.Tensor"
    du: Optional["torch.Tensor"]
    y8: Optional[Packed]        # the output as computed from the kept inputs


class ResidualNorm(NamedTuple):
    x: "torch.Tensor"           # the residual stream behind the block
    h: "torch.Tensor"           # normalised: the next block's input
    stats: "torch.Tensor"       # what the backward call needs of the forward one
    x8: Optional[Packed]
    f8: Optional[Packed]
    h8: Optional[Packed]


class ResidualNormGrads(NamedTuple):
    x: "torch.Tensor"
    f: Optional["torch.Tensor"]
    weight: Optional["torch.Tensor"]
    bias: Optional["torch.Tensor"]
    post_weight: Optional["torch.Tensor"]
    post_bias: Optional["torch.Tensor"]
    gate: Optional["torch.Tensor"]


ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


class UnknownActivation(ValueError, KeyError):
    """A ValueError as for other arguments, and a KeyError for those who look for one."""


def _activation(act) -> int:
    kind = ACTIVATIONS.get(act)
    if kind is None:
        raise UnknownActivation(f"act is one of {', '.join(ACTIVATIONS)}")
    return kind


_pack_rows = struct.Struct("@Pq").pack
_pack_gated = struct.Struct("@qqiiPqPqPqPPP").pack
_pack_norm = struct.Struct("@qqiiiiffiiPPPPPPq").pack
_pack_norm_forward = struct.Struct("@PqPqPqPqPPPP").pack
_pack_norm_backward = struct.Struct("@PqPqPqPqPPPPqPqPqPPPP").pack
_pack_weight_grad = struct.Struct("@qqqiiPqPPqii").pack
_NO_ROWS = (0, 0)


def _matrix(name, t):
    """(tgrad_dtype, rows, width, device index, (address, stride)) of a [rows, width] tensor."""
    types = _torch()[1]
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} is a CUDA tensor [rows, width]")
    d = types.get(t.dtype)
    if d is None or d == C64:
        raise ValueError(f"{name} is fp32, fp16 or bfloat16")
    rows, width = t.shape
    if width < 1:
        raise ValueError(f"{name} has no columns")
    stride, inner = t.stride()
    if (inner != 1 and width > 1) or t.is_neg():
        raise ValueError(f"the entries of a row of {name} are adjacent (and stand there as they are: resolve lazy negations)")
    return d, rows, width, t.get_device(), (t.data_ptr(), stride if rows > 1 else width)


def _like(name, t, d, rows, width, index):
    """(address, stride) of a matrix of the given type, shape and device."""
    m = _matrix(name, t)
    if m[:4] != (d, rows, width, index):
        raise ValueError(f"{name} is a matrix of {rows} x {width} entries, of the others' dtype and device")
    return m[4]


def _packed_bytes(rows, width) -> int:
    blocks = -(-width // 32)
    return rows * (32 * blocks + -(-blocks // 4) * 4)


def _new_packed(rows, width, dtype, index) -> Packed:
    torch = _torch_types[0]
    return Packed(torch.empty(_packed_bytes(rows, width), dtype=torch.uint8, device=index), rows, width, dtype)


def _packed_ptr(name, p, rows, width, dtype, index) -> int:
    """The address of a packed matrix of the given rows, width (None: any), dtype and device."""
    if not isinstance(p, Packed) or p.rows != rows or (width is not None and p.width != width) or p.dtype != dtype:
        raise ValueError(f"{name} is a packed matrix of {rows} x {'any' if width is None else width} entries of {dtype}")
    t = p.data
    if t.dtype is not _torch_types[0].uint8 or not t.is_contiguous() or t.numel() != _packed_bytes(rows, p.width) or not t.is_cuda or t.get_device() != index:
        raise ValueError(f"{name} is not the packed matrix that it says it is, or lives on another device")
    return t.data_ptr()


def act_pack(x, out: Optional[Packed] = None, stream=None) -> Packed:
    """The matrix x in 8.25 bits an entry: 8-bit codes, and a power of two for each block of 32 entries of a row.  An entry reads back
    within half a step, a step being 1/64 of the power of two that its block's largest entry reaches (within one step for an entry that
    near the next power of two).  Zeros and the signs of what does not vanish are kept; a block with an infinity or NaN reads back as NaN.
    `out`: a packed matrix of the same shape and dtype to write to."""
    d, rows, width, index, place = _matrix("x", x)
    if _elsewhere(index, stream):
        return _there(index, stream, act_pack, x, out)
    given = out is not None
    if not given:
        out = _new_packed(rows, width, x.dtype, index)
    to = _packed_ptr("out", out, rows, width, x.dtype, index) if given else out.data.data_ptr()
    _check(lib().tgrad_act_pack(_pack_rows(*place), rows, width, d, to, _raw_stream(index)), "tgrad_act_pack")
    if given:
        _written(out.data)
    return out


def act_unpack(packed: Packed, out=None, stream=None):
    """The matrix that a packed one reads back as, in the dtype that it was packed from."""
    torch, types, _ = _torch()
    if not isinstance(packed, Packed) or not packed.data.is_cuda:
        raise ValueError("packed is a packed matrix on a GPU")
    index = packed.data.get_device()
    if _elsewhere(index, stream):
        return _there(index, stream, act_unpack, packed, out)
    rows, width = packed.rows, packed.width
    src, d = _packed_ptr("packed", packed, rows, width, packed.dtype, index), types.get(packed.dtype)
    if d is None or d == C64:
        raise ValueError("packed is of fp32, fp16 or bfloat16")
    given = out is not None
    if not given:
        out = torch.empty((rows, width), dtype=packed.dtype, device=index)
    _check(lib().tgrad_act_unpack(src, rows, width, d, _pack_rows(*_like("out", out, d, rows, width, index)), _raw_stream(index)), "tgrad_act_unpack")
    if given:
        _written(out)
    return out


def gated_act(a, u=None, act: str = "silu", keep: bool = True, stream=None) -> GatedAct:
    """y = act(a) * u, or act(a) without u, and a and u packed for the backward call (unless keep is False).  act: "silu", "gelu"
    (with the normal distribution) or "gelu_tanh".  a and u may be the halves of one tensor."""
    d, rows, width, index, place = _matrix("a", a)
    if _elsewhere(index, stream):
        return _there(index, stream, gated_act, a, u, act, keep)
    kind = _activation(act)
    other = _like("u", u, d, rows, width, index) if u is not None else _NO_ROWS
    y = _torch_types[0].empty((rows, width), dtype=a.dtype, device=index)
    a8 = _new_packed(rows, width, a.dtype, index) if keep else None
    u8 = _new_packed(rows, width, a.dtype, index) if keep and u is not None else None
    args = _pack_gated(rows, width, d, kind, *place, *other, y.data_ptr(), width, a8.data.data_ptr() if keep else 0, u8.data.data_ptr() if u8 is not None else 0, 0)
    _check(lib().tgrad_gated_act(args, _raw_stream(index)), "tgrad_gated_act")
    return GatedAct(y, a8, u8)


def gated_act_backward(a8: Packed, u8: Optional[Packed], dy, act: str = "silu", keep_y: bool = False, da=None, du=None, stream=None) -> GatedActGrads:
    """Gradients of a gated activation with respect to a and u, from its kept inputs and its output's gradient dy.  keep_y: also the
    output as computed from the kept inputs, packed, the input of the next layer for weight_grad.  `da`, `du`: where to
    write the gradients (such as the halves of one tensor)."""
    d, rows, width, index, place = _matrix("dy", dy)
    if _elsewhere(index, stream):
        return _there(index, stream, gated_act_backward, a8, u8, dy, act, keep_y, da, du)
    kind, given = _activation(act), [t for t in (da, du) if t is not None]
    a_p = _packed_ptr("a8", a8, rows, width, dy.dtype, index)
    u_p = _packed_ptr("u8", u8, rows, width, dy.dtype, index) if u8 is not None else 0
    if u8 is None and du is not None:
        raise ValueError("without u8 there is no du")
    if da is None:
        da = _torch_types[0].empty((rows, width), dtype=dy.dtype, device=index)
    if du is None and u8 is not None:
        du = _torch_types[0].empty((rows, width), dtype=dy.dtype, device=index)
    y8 = _new_packed(rows, width, dy.dtype, index) if keep_y else None
    args = _pack_gated(rows, width, d, kind, *_like("da", da, d, rows, width, index), *(_like("du", du, d, rows, width, index) if du is not None else _NO_ROWS),
                       *place, a_p, u_p, y8.data.data_ptr() if keep_y else 0)
    _check(lib().tgrad_gated_act_backward(args, _raw_stream(index)), "tgrad_gated_act_backward")
    for t in given:
        _written(t)
    return GatedActGrads(da, du, y8)


def _norm_config(d, rows, width, index, weight, bias, post_weight, post_bias, gate, starts, scale, kind, post, eps):
    """(the configuration for the library, tgrad_dtype of the parameters, the gate's rows) after checks of what the library cannot see."""
    torch, types, _ = _torch_types
    if kind not in ("rms", "layer"):
        raise ValueError('kind is "rms" or "layer"')
    if (bias is not None and weight is None) or (post_bias is not None and post_weight is None):
        raise ValueError("a bias comes with its weight")
    params = [("weight", weight), ("bias", bias), ("post_weight", post_weight), ("post_bias", post_bias), ("gate", gate)]
    pd, pointers = None, []
    for name, t in params:
        if t is None:
            pointers.append(0)
            continue
        if pd is None:
            pd = types.get(t.dtype)
        if types.get(t.dtype) != pd or (pd != R32 and pd != d) or t.get_device() != index or not t.is_cuda:
            raise ValueError("parameters are fp32 or of the activations' dtype, all alike, on their device")
        if t.is_neg():
            raise ValueError(f"{name} stands negated: resolve lazy negations")
        if name != "gate" and (t.shape != (width,) or (width > 1 and t.stride(0) != 1)):
            raise ValueError(f"{name} is a contiguous tensor [width]")
        pointers.append(t.data_ptr())
    groups, gate_stride = 0, 0
    if gate is not None:
        if gate.dim() not in (1, 2) or gate.shape[-1] != width or (width > 1 and gate.stride(-1) != 1) or (gate.numel() == 0 and rows > 0):
            raise ValueError("gate is a tensor [width] or [groups, width], the entries of a row adjacent")
        groups, gate_stride = (1, width) if gate.dim() == 1 else (gate.shape[0], gate.stride(0) if gate.shape[0] > 1 else width)
    if starts is not None and (starts.dtype is not torch.int32 or starts.shape != (groups + 1,) or gate is None or not starts.is_cuda or
                               starts.get_device() != index or not starts.is_contiguous()):
        raise ValueError("starts is a contiguous int32 tensor [groups + 1] on the activations' device, and comes with a gate [groups, width]")
    if starts is None and groups and rows % groups:
        raise ValueError("the gate's groups of rows are of equal size unless starts says where they begin")
    if pd is None:
        pd = R32
    return _pack_norm(rows, width, d, pd, kind == "layer", bool(post), scale, eps, groups, 0, starts.data_ptr() if starts is not None and groups else 0,
                      *pointers, gate_stride), pd, groups


def residual_norm(x, f=None, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, starts=None, scale: float = 1.0,
                  kind: str = "rms", post: bool = True, eps: float = 1e-6, keep_x: bool = False, keep_f: bool = False, keep_h: bool = False,
                  stream=None) -> ResidualNorm:
    """The norms around a block's output f, its gate and the residual stream x in one pass:
        x' = scale * x + gate * norm(f; post_weight, post_bias),   h = norm(x'; weight, bias)
    with norm(v) = v / sqrt(mean(v^2) + eps) * weight (kind "rms") or (v - mean) / sqrt(var + eps) * weight + bias ("layer").  post False: f as it is;
    f None: x' = scale * x.  gate: [width], [groups, width] with groups of equal size or those that `starts` (int32 [groups + 1], device) gives, or
    [rows, width]; rows of no group have gate 0, whatever stands in f.  Parameters are fp32 or of x's dtype.  keep_*: x', f or h also packed
    (as rounded), for the backward call or for weight_grad.  Widths up to 16384."""
    d, rows, width, index, place = _matrix("x", x)
    if _elsewhere(index, stream):
        return _there(index, stream, residual_norm, x, f, weight, bias, post_weight, post_bias, gate, starts, scale, kind, post, eps, keep_x, keep_f, keep_h)
    torch, _, f32 = _torch_types
    other = _like("f", f, d, rows, width, index) if f is not None else _NO_ROWS
    if f is None and (gate is not None or post_weight is not None or keep_f):
        raise ValueError("without f there is no gate, no post_weight and nothing of f to keep")
    config, _, _ = _norm_config(d, rows, width, index, weight, bias, post_weight, post_bias, gate, starts, scale, kind, post, eps)
    out, h = (torch.empty((rows, width), dtype=x.dtype, device=index) for _ in range(2))
    stats = torch.empty((4 if kind == "layer" else 2, rows), dtype=f32, device=index)
    kept = [_new_packed(rows, width, x.dtype, index) if k else None for k in (keep_x, keep_f, keep_h)]
    io = _pack_norm_forward(*place, *other, out.data_ptr(), width, h.data_ptr(), width, *(k.data.data_ptr() if k is not None else 0 for k in kept), stats.data_ptr())
    _check(lib().tgrad_residual_norm(config, io, _raw_stream(index)), "tgrad_residual_norm")
    return ResidualNorm(out, h, stats, *kept)


def residual_norm_backward(grad_h, x, stats, f=None, grad_x=None, weight=None, post_weight=None, post_bias=None, gate=None, starts=None,
                           scale: float = 1.0, kind: str = "rms", post: bool = True, stream=None) -> ResidualNormGrads:
    """Gradients of residual_norm from those of h and of x' (grad_x, None: none).  x is the x' that the forward call returned and f its block
    output, each as a tensor or Packed; stats and the other arguments are the forward call's.  Gradients of the parameters that are given (of
    both biases where kind is "layer") have their dtype and shape; sums over rows are fp32, of a fixed order."""
    d, rows, width, index, place = _matrix("grad_h", grad_h)
    if _elsewhere(index, stream):
        return _there(index, stream, residual_norm_backward, grad_h, x, stats, f, grad_x, weight, post_weight, post_bias, gate, starts, scale, kind, post)
    torch, types, f32 = _torch_types
    layer, dtype = kind == "layer", grad_h.dtype

    def either(name, t):
        if t is None:
            return _NO_ROWS, 0
        if isinstance(t, Packed):
            return _NO_ROWS, _packed_ptr(name, t, rows, width, dtype, index)
        return _like(name, t, d, rows, width, index), 0

    (x_m, x_p), (f_m, f_p) = either("x", x), either("f", f)
    if f is None and (gate is not None or post_weight is not None):
        raise ValueError("without f there is no gate and no post_weight")
    g_m = _like("grad_x", grad_x, d, rows, width, index) if grad_x is not None else _NO_ROWS
    if stats.dtype is not f32 or stats.shape != (4 if layer else 2, rows) or stats.get_device() != index or not stats.is_contiguous() or stats.is_neg():
        raise ValueError("stats is what the forward call of the same kind returned")
    config, pd, groups = _norm_config(d, rows, width, index, weight, None, post_weight, post_bias, gate, starts, scale, kind, post, 0.0)
    dx = torch.empty((rows, width), dtype=dtype, device=index)
    df = torch.empty((rows, width), dtype=dtype, device=index) if f is not None else None
    param = dtype if pd == d else f32
    want = [weight is not None, weight is not None and layer, post_weight is not None, post_weight is not None and layer]
    vectors = iter(torch.empty((sum(want), width), dtype=param, device=index).unbind(0))
    dw, db, dpw, dpb = (next(vectors) if k else None for k in want)
    dgate = torch.empty(gate.shape, dtype=param, device=index) if gate is not None else None
    key = ("residual_norm_backward", rows, width, d, pd, layer, groups, starts is not None, index)      # what the workspace's size goes by
    size = _workspace_bytes.get(key)
    if size is None:
        n = C.c_size_t(0)
        _check(lib().tgrad_residual_norm_backward_bytes(config, C.byref(n)), "tgrad_residual_norm_backward_bytes")
        if len(_workspace_bytes) > 4096:
            _workspace_bytes.clear()
        size = _workspace_bytes[key] = n.value
    ws = torch.empty(size, dtype=torch.uint8, device=index)
    io = _pack_norm_backward(*place, *g_m, *x_m, *f_m, x_p, f_p, stats.data_ptr(), dx.data_ptr(), width, df.data_ptr() if df is not None else 0, width,
                             dgate.data_ptr() if dgate is not None else 0, width, *(t.data_ptr() if t is not None else 0 for t in (dw, db, dpw, dpb)))
    _check(lib().tgrad_residual_norm_backward(config, io, ws.data_ptr(), size, _raw_stream(index)), "tgrad_residual_norm_backward")
    return ResidualNormGrads(dx, df, dw, db, dpw, dpb, dgate)


def weight_grad(dy, x8: Packed, dtype=None, out=None, accumulate: bool = False, stream=None):
    """Weight gradient dy^T x [out, width] of a linear layer y = x W^T whose input was kept packed, from its output's gradient dy [rows, out],
    in dy's dtype or fp32 (`dtype`).  `out`: where to write it, or with accumulate what to add it to.  The products are exact;
    sums over 512 tokens (4096 where the result has 16 bits) are the tensor core's, off by at most 2^-17 (2^-14) of the sum of magnitudes, and are
    added in fp32.  dy has the dtype that was packed."""
    d, rows, n, index, place = _matrix("dy", dy)
    if _elsewhere(index, stream):
        return _there(index, stream, weight_grad, dy, x8, dtype, out, accumulate)
    torch, types, f32 = _torch_types
    src = _packed_ptr("x8", x8, rows, None, dy.dtype, index)
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate adds to out")
        out = torch.empty((n, x8.width), dtype=dtype or dy.dtype, device=index)
    to, out_rows, width, where, out_place = _matrix("out", out)
    if (dtype is not None and out.dtype != dtype) or (to != d and to != R32) or (out_rows, width, where) != (n, x8.width, index):
        raise ValueError("out is a matrix [columns of dy, columns of x] of dy's dtype or fp32 on its device")
    args = _pack_weight_grad(rows, n, width, d, to, *place, src, *out_place, accumulate, 0)
    size = C.c_size_t(0)
    _check(lib().tgrad_weight_grad_bytes(args, C.byref(size)), "tgrad_weight_grad_bytes")
    ws = torch.empty(size.value, dtype=torch.uint8, device=index) if size.value else None
    _check(lib().tgrad_weight_grad(args, ws.data_ptr() if ws is not None else 0, size.value, _raw_stream(index)), "tgrad_weight_grad")
    if given:
        _written(out)
    return out

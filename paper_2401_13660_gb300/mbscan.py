"""Python binding of libmbscan.so (argument marshalling only).

Calls on plain, well-formed tensors are marshalled natively (csrc/binding.cpp:
the same checks on the tensors' C++ objects; one mb_step call of one stream 22 -> 3.6 us);
everything else, errors first of all, takes the Python path below it, as does
every call where that module is missing or does not load.

Each function has the name of the C entry point it calls (include/mbscan.h)
and takes torch CUDA tensors in place of device pointers. Every step of the
layer core, and of what a training step runs around it, runs in the library's
kernels; this module only checks tensor shapes/dtypes/devices, fills the C
argument struct and forwards the call on the current torch CUDA stream (or the
stream given). There is no fallback: if the library cannot be loaded, importing
the functions raises.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import threading
import warnings

import torch

from . import build as _build

_lock = threading.Lock()
_lib = None
_fast = None   # csrc/binding.cpp, loaded with the library
# the entry points that binding.cpp calls, in the order of its Api struct
_FAST = ("mb_scan_prefill", "mb_scan_verify", "mb_scan_verify_resume", "mb_scan_prefill_ckpt", "mb_step",
         "mb_step_resume", "mb_rollback", "mb_accept_topk", "mb_rmsnorm", "mb_conv1d_step", "mb_conv_xproj",
         "mb_conv1d", "mb_conv1d_backward", "mb_embed", "mb_embed_backward", "mb_cross_entropy",
         "mb_grad_norm", "mb_grad_clip", "mb_rmsnorm_q8", "mb_quantize_q8", "mb_dequantize_q8", "mb_matmul_q8",
         "mb_sample")

MB_OK, MB_ERR_INVALID_ARG, MB_ERR_UNSUPPORTED, MB_ERR_CUDA, MB_ERR_TIMEOUT = range(5)
MB_F32, MB_BF16 = 0, 1
_DTYPES = {torch.float32: MB_F32, torch.bfloat16: MB_BF16}
_TOKENS = {torch.uint8: 0, torch.int32: 1, torch.int64: 2}


class MbError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {mb_status_string(status)}")


class mb_scan_args(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64),
        ("d_inner", ctypes.c_int64), ("d_state", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("bc_stride", ctypes.c_int32),
        ("x", ctypes.c_void_p), ("z", ctypes.c_void_p), ("dt", ctypes.c_void_p),
        ("B", ctypes.c_void_p), ("C", ctypes.c_void_p),
        ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p),
        ("h0", ctypes.c_void_p), ("y", ctypes.c_void_p),
        ("dt_low", ctypes.c_void_p), ("W_dt", ctypes.c_void_p),
        ("dt_rank", ctypes.c_int32), ("dt_low_stride", ctypes.c_int32),
    ]


class mb_scan_grads(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dz", ctypes.c_void_p), ("ddt", ctypes.c_void_p),
                ("dB", ctypes.c_void_p), ("dC", ctypes.c_void_p), ("dA", ctypes.c_void_p),
                ("dD", ctypes.c_void_p), ("ddt_bias", ctypes.c_void_p), ("dh0", ctypes.c_void_p)]


class mb_conv1d_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64), ("width", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("x_stride", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("state", ctypes.c_void_p),
                ("w", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


class mb_conv1d_grads(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dx_stride", ctypes.c_int64), ("dstate", ctypes.c_void_p),
                ("dw", ctypes.c_void_p), ("dbias", ctypes.c_void_p)]


class mb_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


MB_CKPT_STEPS = 16


class _Declined:
    """Stands in for the native marshalling where it cannot be had: every call takes the Python path."""

    def __getattr__(self, name):
        return lambda *a: -1


def _load_binding(lib):
    try:
        loader = importlib.machinery.ExtensionFileLoader("_mbcall", _build.BINDING)
        fast = importlib.util.module_from_spec(importlib.util.spec_from_file_location(
            "_mbcall", _build.BINDING, loader=loader))
        loader.exec_module(fast)
        fast.init(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _FAST))
        return fast
    except ImportError as e:
        warnings.warn(f"native argument marshalling not loaded, calls are marshalled in Python: {e}")
        return _Declined()


def library_path() -> str:
    return _build.LIB


def load_library(build_if_needed: bool = True) -> ctypes.CDLL:
    """Load libmbscan.so (building it first if it is missing or stale)."""
    global _lib, _fast
    with _lock:
        if _lib is None:
            path = _build.build() if build_if_needed else _build.LIB
            if not os.path.exists(path):
                raise RuntimeError(f"libmbscan.so not found at {path}; run build() first")
            lib = ctypes.CDLL(path)
            vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
            ap = ctypes.POINTER(mb_scan_args)
            lib.mb_workspace_size.argtypes = [ap]
            lib.mb_workspace_size.restype = sz
            lib.mb_scan_prefill.argtypes = [ap, vp, vp, sz, vp]
            lib.mb_scan_verify.argtypes = [ap, vp, vp, sz, vp]
            lib.mb_rollback.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, vp]
            lib.mb_step.argtypes = [ap, vp, vp, sz, vp]
            lib.mb_check.argtypes = [vp, vp, ctypes.POINTER(i64)]
            lib.mb_accept_topk.argtypes = [vp, ctypes.c_int32, vp, i64, i64, ctypes.c_int32, vp, vp]
            lib.mb_step_resume.argtypes = [ap, vp, vp, i64, vp, vp, sz, vp]
            lib.mb_scan_prefill_ckpt.argtypes = [ap, vp, vp, vp, sz, vp]
            lib.mb_rmsnorm.argtypes = [vp, vp, vp, ctypes.c_float, vp, i64, i64, ctypes.c_int32, vp]
            lib.mb_conv1d_step.argtypes = [vp, vp, vp, vp, vp, i64, i64, ctypes.c_int32, vp]
            lib.mb_scan_backward.argtypes = [ap, vp, vp, vp, ctypes.POINTER(mb_scan_grads), vp, sz, vp]
            lib.mb_selftest_timeout.argtypes = [vp, sz, i64, vp]
            lib.mb_scan_verify_resume.argtypes = [ap, vp, vp, i64, vp, vp, sz, vp]
            lib.mb_conv_xproj_workspace_size.argtypes = [i64, i64, ctypes.c_int32]
            lib.mb_conv_xproj_workspace_size.restype = sz
            lib.mb_conv_xproj.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, ctypes.c_int32, ctypes.c_int32,
                                          vp, sz, vp]
            cp = ctypes.POINTER(mb_conv1d_args)
            lib.mb_conv1d.argtypes = [cp, vp, vp, vp]
            lib.mb_conv1d_backward_workspace_size.argtypes = [i64, i64, i64]
            lib.mb_conv1d_backward_workspace_size.restype = sz
            lib.mb_conv1d_backward.argtypes = [cp, vp, vp, ctypes.POINTER(mb_conv1d_grads), vp, sz, vp]
            i32, f32 = ctypes.c_int32, ctypes.c_float
            lib.mb_embed.argtypes = [vp, i32, vp, i32, f32, vp, i32, i64, i64, i64, vp]
            lib.mb_embed_backward_workspace_size.argtypes = [i64, i64, i64]
            lib.mb_embed_backward_workspace_size.restype = sz
            lib.mb_embed_backward.argtypes = [vp, i32, vp, i32, f32, i32, vp, i64, i64, i64, vp, sz, vp]
            lib.mb_cross_entropy.argtypes = [vp, i32, vp, i32, vp, f32, vp, vp, i64, i64, vp]
            lib.mb_grad_norm_workspace_size.argtypes = []
            lib.mb_grad_norm_workspace_size.restype = sz
            tp = ctypes.POINTER(mb_tensor)
            lib.mb_grad_norm.argtypes = [tp, i64, vp, vp, sz, vp]
            lib.mb_grad_clip.argtypes = [tp, tp, i64, vp, f32, vp]
            lib.mb_q8_scale_stride.argtypes = [i64]
            lib.mb_q8_scale_stride.restype = i64
            lib.mb_rmsnorm_q8.argtypes = [vp, i32, vp, vp, f32, vp, vp, i64, i64, vp]
            lib.mb_quantize_q8.argtypes = [vp, i32, i64, i32, vp, vp, i64, i64, vp]
            lib.mb_dequantize_q8.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp]
            lib.mb_matmul_q8.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, i64, vp, sz, vp]
            lib.mb_matmul_q8_form.argtypes = [i64, i64, i64, i32, ctypes.POINTER(i64)]
            lib.mb_sample.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, i64, i64, vp]
            for f in ("mb_scan_prefill", "mb_scan_verify", "mb_rollback", "mb_step", "mb_check",
                      "mb_accept_topk", "mb_step_resume", "mb_scan_prefill_ckpt", "mb_scan_backward",
                      "mb_rmsnorm", "mb_conv1d_step", "mb_selftest_timeout", "mb_scan_verify_resume",
                      "mb_conv_xproj", "mb_conv1d", "mb_conv1d_backward", "mb_embed", "mb_embed_backward",
                      "mb_cross_entropy", "mb_grad_norm", "mb_grad_clip", "mb_rmsnorm_q8", "mb_quantize_q8",
                      "mb_dequantize_q8", "mb_matmul_q8", "mb_matmul_q8_form", "mb_sample"):
                getattr(lib, f).restype = ctypes.c_int
            lib.mb_status_string.argtypes = [ctypes.c_int]
            lib.mb_status_string.restype = ctypes.c_char_p
            lib.mb_version.argtypes = []
            lib.mb_version.restype = ctypes.c_char_p
            _fast = _load_binding(lib)
            _lib = lib
    return _lib


def _native():
    load_library()
    return _fast


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream, dev):
    """The stream of a call whose tensors are on `dev`. Every launch asks here: host memory's addresses go no further."""
    if dev.type != "cuda":
        raise ValueError(f"tensors on {dev}, expected a CUDA device")
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _need(t, name, dtype=None, shape=None, device=None):
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def _row_stride(name, t, batch, L, width, dtype, dev):
    """Row stride (elements) of t [batch, L, width]: width when contiguous,
    or S when t is a column block of wider rows (strides (L*S, S, 1))."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype or tuple(t.shape) != (batch, L, width) or t.device != dev:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtype} "
                         f"{(batch, L, width)} on {dev}")
    if t.is_contiguous():
        return width
    sb, st, sn = t.stride()
    if sn != 1 or (L > 1 and sb != L * st) or st < width:
        raise ValueError(f"{name} must be contiguous or have strides (L*S, S, 1)")
    return st if L > 1 or batch == 1 else sb


def _bc_row_stride(B, C, batch, L, N, dtype, dev):
    """Row stride (elements) shared by B and C [batch, L, N]: N for
    contiguous tensors, or S when both are column blocks of wider rows
    (strides (L*S, S, 1))."""
    strides = {_row_stride(name, t, batch, L, N, dtype, dev) for name, t in (("B", B), ("C", C))}
    if len(strides) != 1:
        raise ValueError("B and C must share one row stride")
    return strides.pop()


def make_args(x, dt, B, C, A, y, *, z=None, D=None, dt_bias=None, h0=None, dt_low=None,
              W_dt=None) -> mb_scan_args:
    """Fill mb_scan_args from tensors. x, dt, z, y: [batch, L, d_inner];
    B, C: [batch, L, d_state] (all one dtype, fp32 or bf16), contiguous or
    column blocks of wider rows (strides (L*S, S, 1): bc_stride = S); A:
    [d_inner, d_state], D, dt_bias: [d_inner], h0: [batch, d_inner, d_state]
    (fp32). Fused Delta projection: dt = None, dt_low [batch, L, r] (contiguous
    or a column block of wider rows) and W_dt [d_inner, r]; the kernels then
    form dt = dt_low W_dt^T themselves."""
    if x.dtype not in _DTYPES:
        raise TypeError(f"unsupported input dtype {x.dtype}")
    batch, L, Dn = x.shape
    N = A.shape[1]
    dev = x.device
    if (dt is None) == (dt_low is None):
        raise ValueError("pass exactly one of dt and dt_low")
    if dt_low is not None and W_dt is None:
        raise ValueError("dt_low needs W_dt")
    for name, t in (("x", x), ("dt", dt), ("z", z), ("y", y)):
        _need(t, name, x.dtype, (batch, L, Dn), dev)
    S = _bc_row_stride(B, C, batch, L, N, x.dtype, dev)
    _need(A, "A", torch.float32, (Dn, N), dev)
    _need(D, "D", torch.float32, (Dn,), dev)
    _need(dt_bias, "dt_bias", torch.float32, (Dn,), dev)
    _need(h0, "h0", torch.float32, (batch, Dn, N), dev)
    a = mb_scan_args()
    a.batch, a.seqlen, a.d_inner, a.d_state = batch, L, Dn, N
    a.dtype = _DTYPES[x.dtype]
    a.bc_stride = 0 if S == N else S
    if dt_low is not None:
        r = W_dt.shape[1] if W_dt.dim() == 2 else -1
        _need(W_dt, "W_dt", x.dtype, (Dn, r), dev)
        S = _row_stride("dt_low", dt_low, batch, L, r, x.dtype, dev)
        a.dt_low, a.W_dt = dt_low.data_ptr(), W_dt.data_ptr()
        a.dt_rank = r
        a.dt_low_stride = 0 if S == r else S
    a.x, a.z, a.dt, a.B, a.C = (t.data_ptr() if t is not None else None for t in (x, z, dt, B, C))
    a.A, a.D, a.dt_bias, a.h0 = (t.data_ptr() if t is not None else None for t in (A, D, dt_bias, h0))
    a.y = y.data_ptr()
    return a


def _check(rc, where):
    if rc != MB_OK:
        raise MbError(rc, where)


def mb_status_string(status: int) -> str:
    return load_library().mb_status_string(int(status)).decode()


def mb_version() -> str:
    return load_library().mb_version().decode()


def mb_workspace_size(args: mb_scan_args) -> int:
    return int(load_library().mb_workspace_size(ctypes.byref(args)))


def new_workspace(args: mb_scan_args, device) -> torch.Tensor:
    """Zeroed workspace tensor for `args` (uint8, 256-byte aligned by torch)."""
    n = max(mb_workspace_size(args), 256)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def mb_scan_prefill(x, dt, B, C, A, y, *, z=None, D=None, dt_bias=None, h0=None, h_last=None,
                    ws=None, stream=None, dt_low=None, W_dt=None):
    """Prefill scan: writes y and (if given) h_last [batch, d_inner, d_state].
    dt = None with dt_low, W_dt: the fused Delta projection (see make_args)."""
    if ws is not None and stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).prefill(x, dt, B, C, A, y, z, D, dt_bias, h0, h_last, ws)
        if rc >= 0:
            _check(rc, "mb_scan_prefill")
            return y, h_last
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, h0=h0, dt_low=dt_low, W_dt=W_dt)
    _need(h_last, "h_last", torch.float32, (a.batch, a.d_inner, a.d_state), x.device)
    if ws is None:
        ws = new_workspace(a, x.device)
    rc = load_library().mb_scan_prefill(ctypes.byref(a), _ptr(h_last), _ptr(ws), ws.numel(),
                                        _stream(stream, x.device))
    _check(rc, "mb_scan_prefill")
    return y, h_last


def mb_scan_verify(x, dt, B, C, A, y, h_all, *, z=None, D=None, dt_bias=None, h0=None, ws=None,
                   stream=None, dt_low=None, W_dt=None):
    """Verify scan of k = x.shape[1] drafted bytes: y and h_all [batch, k, d_inner, d_state]."""
    if ws is not None and stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).verify(x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, ws)
        if rc >= 0:
            _check(rc, "mb_scan_verify")
            return y, h_all
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, h0=h0, dt_low=dt_low, W_dt=W_dt)
    _need(h_all, "h_all", torch.float32, (a.batch, a.seqlen, a.d_inner, a.d_state), x.device)
    if ws is None:
        ws = new_workspace(a, x.device)
    rc = load_library().mb_scan_verify(ctypes.byref(a), _ptr(h_all), _ptr(ws), ws.numel(),
                                       _stream(stream, x.device))
    _check(rc, "mb_scan_verify")
    return y, h_all


def mb_scan_verify_resume(x, dt, B, C, A, y, h_all, h_all_prev, accept, *, z=None, D=None, dt_bias=None,
                          h0=None, ws=None, stream=None, dt_low=None, W_dt=None):
    """Verify of k = x.shape[1] drafted bytes, stream s starting from h0[s]
    (zeros if None) when accept[s] == 0, else from h_all_prev[s, accept[s]-1]
    (the previous verify's per-position states, [batch, k_prev, d_inner,
    d_state]). A bad accept count is recorded in ws (mb_check) and that stream
    is left untouched."""
    if ws is not None and stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).verify_resume(x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, h_all_prev, accept, ws)
        if rc >= 0:
            _check(rc, "mb_scan_verify_resume")
            return y, h_all
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, h0=h0, dt_low=dt_low, W_dt=W_dt)
    _need(h_all, "h_all", torch.float32, (a.batch, a.seqlen, a.d_inner, a.d_state), x.device)
    _need(h_all_prev, "h_all_prev", torch.float32, None, x.device)
    if h_all_prev.dim() != 4 or h_all_prev.shape[0] != a.batch or \
            tuple(h_all_prev.shape[2:]) != (a.d_inner, a.d_state):
        raise ValueError(f"h_all_prev: shape {tuple(h_all_prev.shape)}, expected [batch, k_prev, d_inner, d_state]")
    _need(accept, "accept", torch.int32, (a.batch,), x.device)
    if ws is None:
        ws = new_workspace(a, x.device)
    rc = load_library().mb_scan_verify_resume(ctypes.byref(a), _ptr(h_all_prev), _ptr(accept), h_all_prev.shape[1],
                                              _ptr(h_all), _ptr(ws), ws.numel(), _stream(stream, x.device))
    _check(rc, "mb_scan_verify_resume")
    return y, h_all


def mb_rollback(h0, h_all, accept, h_out, *, ws=None, stream=None):
    """h_out[s] = h0[s] if accept[s] == 0 else h_all[s, accept[s]-1]."""
    if stream is None:
        rc = (_fast or _native()).rollback(h0, h_all, accept, h_out, ws)
        if rc >= 0:
            _check(rc, "mb_rollback")
            return h_out
    batch, k, Dn, N = h_all.shape
    _need(h_all, "h_all", torch.float32)
    _need(h0, "h0", torch.float32, (batch, Dn, N), h_all.device)
    _need(h_out, "h_out", torch.float32, (batch, Dn, N), h_all.device)
    _need(accept, "accept", torch.int32, (batch,), h_all.device)
    rc = load_library().mb_rollback(_ptr(h0), _ptr(h_all), _ptr(accept), _ptr(h_out), batch, k,
                                    Dn, N, _ptr(ws), _stream(stream, h_all.device))
    _check(rc, "mb_rollback")
    return h_out


def mb_step(x, dt, B, C, A, y, state, *, z=None, D=None, dt_bias=None, ws=None, stream=None, dt_low=None,
            W_dt=None):
    """One decode step: x, dt, z, y [batch, 1, d_inner]; B, C [batch, 1, d_state];
    state [batch, d_inner, d_state] updated in place. ws (optional, >= 256
    bytes): status block where a timed-out wait is recorded (mb_check)."""
    if stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).step(x, dt, B, C, A, y, z, D, dt_bias, None, state, ws)
        if rc >= 0:
            _check(rc, "mb_step")
            return y, state
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, dt_low=dt_low, W_dt=W_dt)
    _need(state, "state", torch.float32, (a.batch, a.d_inner, a.d_state), x.device)
    _need(ws, "ws", torch.uint8, None, x.device)
    nbytes = 0 if ws is None else ws.numel()
    rc = load_library().mb_step(ctypes.byref(a), _ptr(state), _ptr(ws), nbytes, _stream(stream, x.device))
    _check(rc, "mb_step")
    return y, state


def mb_scan_prefill_ckpt(x, dt, B, C, A, y, h_ckpt=None, *, z=None, D=None, dt_bias=None, h0=None,
                         h_last=None, ws=None, stream=None, dt_low=None, W_dt=None):
    """Training forward: prefill that also writes h_ckpt [batch, ceil(L / 16),
    d_inner, d_state], the state before every 16-step chunk (allocated when
    None). Returns (y, h_last, h_ckpt). (The fused Delta projection is not
    accepted here: MB_ERR_UNSUPPORTED.)"""
    if ws is not None and h_ckpt is not None and stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).prefill_ckpt(x, dt, B, C, A, y, z, D, dt_bias, h0, h_last, h_ckpt, ws)
        if rc >= 0:
            _check(rc, "mb_scan_prefill_ckpt")
            return y, h_last, h_ckpt
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, h0=h0, dt_low=dt_low, W_dt=W_dt)
    nch = (a.seqlen + MB_CKPT_STEPS - 1) // MB_CKPT_STEPS
    if h_ckpt is None:
        h_ckpt = torch.empty(a.batch, nch, a.d_inner, a.d_state, dtype=torch.float32, device=x.device)
    _need(h_ckpt, "h_ckpt", torch.float32, (a.batch, nch, a.d_inner, a.d_state), x.device)
    _need(h_last, "h_last", torch.float32, (a.batch, a.d_inner, a.d_state), x.device)
    if ws is None:
        ws = new_workspace(a, x.device)
    rc = load_library().mb_scan_prefill_ckpt(ctypes.byref(a), _ptr(h_last), _ptr(h_ckpt), _ptr(ws),
                                             ws.numel(), _stream(stream, x.device))
    _check(rc, "mb_scan_prefill_ckpt")
    return y, h_last, h_ckpt


def mb_scan_backward(x, dt, B, C, A, h_ckpt, dout, *, z=None, D=None, dt_bias=None, h0=None,
                     dh_last=None, grads=None, ws=None, stream=None):
    """Backward of the layer core. Returns a dict of gradients: dx, ddt, dz (or
    None) in the input dtype [batch, L, d_inner]; dB, dC fp32 [batch, L,
    d_state]; dA fp32 [d_inner, d_state]; dD, ddt_bias fp32 [d_inner]; dh0 fp32
    [batch, d_inner, d_state]. Tensors missing from `grads` are allocated."""
    if x.dtype not in _DTYPES:
        raise TypeError(f"unsupported input dtype {x.dtype}")
    batch, L, Dn = x.shape
    N = A.shape[1]
    dev = x.device
    a = make_args(x, dt, B, C, A, x, z=z, D=D, dt_bias=dt_bias, h0=h0)
    a.y = None
    nch = (L + MB_CKPT_STEPS - 1) // MB_CKPT_STEPS
    _need(h_ckpt, "h_ckpt", torch.float32, (batch, nch, Dn, N), dev)
    _need(dout, "dout", x.dtype, (batch, L, Dn), dev)
    _need(dh_last, "dh_last", torch.float32, (batch, Dn, N), dev)
    g = dict(grads or {})
    shapes = {"dx": ((batch, L, Dn), x.dtype), "ddt": ((batch, L, Dn), x.dtype),
              "dz": ((batch, L, Dn), x.dtype), "dB": ((batch, L, N), torch.float32),
              "dC": ((batch, L, N), torch.float32), "dA": ((Dn, N), torch.float32),
              "dD": ((Dn,), torch.float32), "ddt_bias": ((Dn,), torch.float32),
              "dh0": ((batch, Dn, N), torch.float32)}
    for k, (shp, dty) in shapes.items():
        if k == "dz" and z is None:
            g[k] = None
            continue
        if g.get(k) is None:
            g[k] = torch.empty(shp, dtype=dty, device=dev)
        _need(g[k], k, dty, shp, dev)
    st = mb_scan_grads(*(None if g[k] is None else g[k].data_ptr() for k in
                         ("dx", "dz", "ddt", "dB", "dC", "dA", "dD", "ddt_bias", "dh0")))
    if ws is None:
        ws = new_workspace(a, dev)
    rc = load_library().mb_scan_backward(ctypes.byref(a), _ptr(h_ckpt), _ptr(dout), _ptr(dh_last),
                                         ctypes.byref(st), _ptr(ws), ws.numel(), _stream(stream, dev))
    _check(rc, "mb_scan_backward")
    return g


def mb_rmsnorm(residual, w, out, *, add=None, eps=1e-5, stream=None):
    """residual [batch, width] fp32 += add (if given); out = residual * w /
    rms(residual), out and add in the input dtype (fp32 or bf16)."""
    if stream is None:
        rc = (_fast or _native()).rmsnorm(residual, w, out, add, eps)
        if rc >= 0:
            _check(rc, "mb_rmsnorm")
            return out
    if out.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {out.dtype}")
    batch, width = residual.shape
    dev = residual.device
    _need(residual, "residual", torch.float32, (batch, width), dev)
    _need(w, "w", torch.float32, (width,), dev)
    _need(out, "out", out.dtype, (batch, width), dev)
    _need(add, "add", out.dtype, (batch, width), dev)
    rc = load_library().mb_rmsnorm(_ptr(add), _ptr(residual), _ptr(w), float(eps), _ptr(out), batch, width,
                                   _DTYPES[out.dtype], _stream(stream, dev))
    _check(rc, "mb_rmsnorm")
    return out


def mb_conv1d_step(x, state, w, out, *, bias=None, stream=None):
    """One causal depthwise convolution step (kernel 4) with SiLU: x, out
    [batch, width]; state [batch, 3, width] (previous inputs, oldest first),
    updated in place; w [width, 4] fp32; bias [width] fp32."""
    if stream is None:
        rc = (_fast or _native()).conv1d_step(x, state, w, out, bias)
        if rc >= 0:
            _check(rc, "mb_conv1d_step")
            return out
    if x.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {x.dtype}")
    batch, width = x.shape
    dev = x.device
    _need(x, "x", x.dtype, (batch, width), dev)
    _need(state, "state", x.dtype, (batch, 3, width), dev)
    _need(w, "w", torch.float32, (width, 4), dev)
    _need(bias, "bias", torch.float32, (width,), dev)
    _need(out, "out", x.dtype, (batch, width), dev)
    rc = load_library().mb_conv1d_step(_ptr(x), _ptr(state), _ptr(w), _ptr(bias), _ptr(out), batch, width,
                                       _DTYPES[x.dtype], _stream(stream, dev))
    _check(rc, "mb_conv1d_step")
    return out


def mb_conv_xproj_workspace_size(batch: int, width: int, n_out: int) -> int:
    """Workspace bytes mb_conv_xproj needs (0: shape not supported)."""
    return int(load_library().mb_conv_xproj_workspace_size(batch, width, n_out))


def mb_conv_xproj(x, state, w, W, xc, out, ws, *, bias=None, stream=None):
    """Convolution step fused with the x-projection: xc = silu(conv1d_step(x))
    as mb_conv1d_step (state [batch, 3, width] updated in place), then
    out = xc W^T. x, xc [batch, width], W [n_out, width], out [batch, n_out],
    all bf16; w [width, 4], bias [width] fp32; ws a uint8 workspace of
    mb_conv_xproj_workspace_size bytes."""
    if stream is None:
        rc = (_fast or _native()).conv_xproj(x, state, w, W, xc, out, ws, bias)
        if rc >= 0:
            _check(rc, "mb_conv_xproj")
            return out
    batch, width = x.shape
    n_out = W.shape[0]
    dev, bf = x.device, torch.bfloat16
    _need(x, "x", bf, (batch, width), dev)
    _need(state, "state", bf, (batch, 3, width), dev)
    _need(w, "w", torch.float32, (width, 4), dev)
    _need(bias, "bias", torch.float32, (width,), dev)
    _need(W, "W", bf, (n_out, width), dev)
    _need(xc, "xc", bf, (batch, width), dev)
    _need(out, "out", bf, (batch, n_out), dev)
    _need(ws, "ws", torch.uint8, None, dev)
    rc = load_library().mb_conv_xproj(_ptr(x), _ptr(state), _ptr(w), _ptr(bias), _ptr(W), _ptr(xc), _ptr(out),
                                      batch, width, n_out, MB_BF16, _ptr(ws), ws.numel(), _stream(stream, x.device))
    _check(rc, "mb_conv_xproj")
    return out


def mb_step_resume(x, dt, B, C, A, y, h_all, accept, state, *, z=None, D=None, dt_bias=None, h0=None,
                   ws=None, stream=None, dt_low=None, W_dt=None):
    """One decode step from the state kept after accept[s] drafted bytes:
    h0[s] (zeros if None) when accept[s] == 0, else h_all[s, accept[s]-1].
    x, dt, z, y [batch, 1, d_inner]; B, C [batch, 1, d_state]; h_all [batch,
    k, d_inner, d_state]; accept [batch] int32; state [batch, d_inner,
    d_state] is written (it may be h0 itself)."""
    if stream is None and dt_low is None and W_dt is None:
        rc = (_fast or _native()).step_resume(x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, accept, state, ws)
        if rc >= 0:
            _check(rc, "mb_step_resume")
            return y, state
    a = make_args(x, dt, B, C, A, y, z=z, D=D, dt_bias=dt_bias, h0=h0, dt_low=dt_low, W_dt=W_dt)
    _need(h_all, "h_all", torch.float32, None, x.device)
    if h_all.dim() != 4 or h_all.shape[0] != a.batch or tuple(h_all.shape[2:]) != (a.d_inner, a.d_state):
        raise ValueError(f"h_all: shape {tuple(h_all.shape)}, expected [batch, k, d_inner, d_state]")
    _need(accept, "accept", torch.int32, (a.batch,), x.device)
    _need(state, "state", torch.float32, (a.batch, a.d_inner, a.d_state), x.device)
    nbytes = 0 if ws is None else ws.numel()
    rc = load_library().mb_step_resume(ctypes.byref(a), _ptr(h_all), _ptr(accept), h_all.shape[1],
                                       _ptr(state), _ptr(ws), nbytes, _stream(stream, x.device))
    _check(rc, "mb_step_resume")
    return y, state


def mb_accept_topk(logits, drafted, beta, accept=None, stream=None):
    """Accept counts of speculative decoding: logits [streams, k, 256] (fp32 or
    bf16), drafted [streams, k] uint8 -> accept [streams] int32."""
    if accept is not None and stream is None:
        rc = (_fast or _native()).accept_topk(logits, drafted, accept, beta)
        if rc >= 0:
            _check(rc, "mb_accept_topk")
            return accept
    if logits.dtype not in _DTYPES:
        raise TypeError(f"unsupported logits dtype {logits.dtype}")
    streams, k, v = logits.shape
    if v != 256:
        raise ValueError("logits must have 256 entries per position")
    _need(logits, "logits", logits.dtype)
    _need(drafted, "drafted", torch.uint8, (streams, k), logits.device)
    if accept is None:
        accept = torch.empty(streams, dtype=torch.int32, device=logits.device)
    _need(accept, "accept", torch.int32, (streams,), logits.device)
    rc = load_library().mb_accept_topk(_ptr(logits), _DTYPES[logits.dtype], _ptr(drafted), streams, k,
                                       int(beta), _ptr(accept), _stream(stream, logits.device))
    _check(rc, "mb_accept_topk")
    return accept


def _conv1d_args(x, w, bias, state) -> mb_conv1d_args:
    if x.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {x.dtype}")
    batch, L, width = x.shape
    dev = x.device
    S = _row_stride("x", x, batch, L, width, x.dtype, dev)
    _need(w, "w", torch.float32, (width, 4), dev)
    _need(bias, "bias", torch.float32, (width,), dev)
    _need(state, "state", x.dtype, (batch, 3, width), dev)
    if S > 0x7fffffff:
        raise ValueError(f"x: rows {S} elements apart, at most 2^31 - 1")
    a = mb_conv1d_args()
    a.batch, a.seqlen, a.width, a.dtype = batch, L, width, _DTYPES[x.dtype]
    a.x_stride = 0 if S == width else S
    a.x, a.state, a.w, a.bias = (t.data_ptr() if t is not None else None for t in (x, state, w, bias))
    return a


def mb_conv1d(x, w, out, *, bias=None, state=None, state_out=None, stream=None):
    """Causal depthwise convolution (kernel 4) with SiLU over a span: x
    [batch, L, width] (contiguous or a column block of wider rows, strides
    (L*S, S, 1)), out [batch, L, width]; w [width, 4], bias [width] fp32; state
    [batch, 3, width]: the inputs before the span, oldest first (None: zeros);
    state_out (if given): those before the next one, as mb_conv1d_step's state
    (it may be `state` itself)."""
    if stream is None:
        rc = (_fast or _native()).conv1d(x, w, out, bias, state, state_out)
        if rc >= 0:
            _check(rc, "mb_conv1d")
            return out
    a = _conv1d_args(x, w, bias, state)
    _need(out, "out", x.dtype, tuple(x.shape), x.device)
    _need(state_out, "state_out", x.dtype, (a.batch, 3, a.width), x.device)
    rc = load_library().mb_conv1d(ctypes.byref(a), _ptr(out), _ptr(state_out), _stream(stream, x.device))
    _check(rc, "mb_conv1d")
    return out


def mb_conv1d_backward_workspace_size(batch: int, seqlen: int, width: int) -> int:
    """Workspace bytes mb_conv1d_backward needs (0: sizes not accepted)."""
    return int(load_library().mb_conv1d_backward_workspace_size(batch, seqlen, width))


def mb_conv1d_backward(x, w, dout, *, bias=None, state=None, dstate_out=None, grads=None, ws=None, stream=None):
    """Gradients of mb_conv1d given dout [batch, L, width] and dstate_out
    [batch, 3, width] (None: zeros). Returns a dict: dx [batch, L, width]
    (`grads["dx"]` may be a column block of wider rows), dw [width, 4] fp32,
    dbias [width] fp32 (None without a bias, unless given), dstate [batch, 3,
    width] (None without a state, unless given). What is missing from `grads`
    is allocated, and ws too."""
    wanted = {"dx": True, "dw": True, "dbias": bias is not None, "dstate": state is not None}
    g = {k: (grads or {}).get(k) for k in wanted}
    if ws is not None and stream is None and all(g[k] is not None for k, want in wanted.items() if want):
        rc = (_fast or _native()).conv1d_backward(x, w, dout, bias, state, dstate_out, g["dx"], g["dw"], g["dbias"],
                                                  g["dstate"], ws)
        if rc >= 0:
            _check(rc, "mb_conv1d_backward")
            return g
    a = _conv1d_args(x, w, bias, state)
    batch, L, width = x.shape
    dev = x.device
    _need(dout, "dout", x.dtype, (batch, L, width), dev)
    _need(dstate_out, "dstate_out", x.dtype, (batch, 3, width), dev)
    shapes = {"dx": ((batch, L, width), x.dtype), "dw": ((width, 4), torch.float32),
              "dbias": ((width,), torch.float32), "dstate": ((batch, 3, width), x.dtype)}
    for k, (shape, dtype) in shapes.items():
        if g[k] is None and wanted[k]:
            g[k] = torch.empty(shape, dtype=dtype, device=dev)
        if k != "dx":
            _need(g[k], k, dtype, shape, dev)
    S = _row_stride("dx", g["dx"], batch, L, width, x.dtype, dev)
    st = mb_conv1d_grads(g["dx"].data_ptr(), 0 if S == width else S,
                         *(None if g[k] is None else g[k].data_ptr() for k in ("dstate", "dw", "dbias")))
    if ws is None:
        ws = torch.zeros(max(mb_conv1d_backward_workspace_size(batch, L, width), 256), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8, None, dev)
    rc = load_library().mb_conv1d_backward(ctypes.byref(a), _ptr(dout), _ptr(dstate_out), ctypes.byref(st), _ptr(ws),
                                           ws.numel(), _stream(stream, dev))
    _check(rc, "mb_conv1d_backward")
    return g


def _token_type(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in _TOKENS:
        raise TypeError(f"{name}: dtype {t.dtype}, expected one of {list(_TOKENS)}")
    return _TOKENS[t.dtype]


def mb_embed(tokens, table, out, *, scale=1.0, stream=None):
    """out[..., :] = scale * table[tokens] (zeros where a token is outside the
    table): tokens uint8, int32 or int64, any shape; table [vocab, width]; out
    [*tokens.shape, width]; table and out fp32 or bf16 each."""
    if stream is None:
        rc = (_fast or _native()).embed(tokens, table, out, scale)
        if rc >= 0:
            _check(rc, "mb_embed")
            return out
    tt = _token_type(tokens, "tokens")
    for name, t in (("table", table), ("out", out)):
        if t.dtype not in _DTYPES:
            raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    vocab, width = table.shape
    dev = table.device
    _need(tokens, "tokens", None, None, dev)
    _need(table, "table")
    _need(out, "out", None, (*tokens.shape, width), dev)
    rc = load_library().mb_embed(_ptr(tokens), tt, _ptr(table), _DTYPES[table.dtype], float(scale), _ptr(out),
                                 _DTYPES[out.dtype], tokens.numel(), vocab, width, _stream(stream, dev))
    _check(rc, "mb_embed")
    return out


def mb_embed_backward_workspace_size(n: int, vocab: int, width: int) -> int:
    """Workspace bytes mb_embed_backward needs for n tokens (0: sizes not accepted)."""
    return int(load_library().mb_embed_backward_workspace_size(n, vocab, width))


def mb_embed_backward(tokens, dout, dtable, *, scale=1.0, accumulate=False, ws=None, stream=None):
    """dtable [vocab, width] fp32 = (accumulate: itself +) scale * the sum of
    dout's rows for each token: tokens as in mb_embed, dout [*tokens.shape,
    width] fp32 or bf16."""
    if ws is not None and stream is None:
        rc = (_fast or _native()).embed_backward(tokens, dout, dtable, scale, accumulate, ws)
        if rc >= 0:
            _check(rc, "mb_embed_backward")
            return dtable
    tt = _token_type(tokens, "tokens")
    if dout.dtype not in _DTYPES:
        raise TypeError(f"dout: unsupported dtype {dout.dtype}")
    vocab, width = dtable.shape
    dev = dtable.device
    _need(tokens, "tokens", None, None, dev)
    _need(dtable, "dtable", torch.float32)
    _need(dout, "dout", None, (*tokens.shape, width), dev)
    n = tokens.numel()
    if ws is None:
        ws = torch.zeros(max(mb_embed_backward_workspace_size(n, vocab, width), 256), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8, None, dev)
    rc = load_library().mb_embed_backward(_ptr(tokens), tt, _ptr(dout), _DTYPES[dout.dtype], float(scale),
                                          int(bool(accumulate)), _ptr(dtable), n, vocab, width, _ptr(ws), ws.numel(),
                                          _stream(stream, dev))
    _check(rc, "mb_embed_backward")
    return dtable


def mb_cross_entropy(logits, targets, loss, dlogits=None, *, weight=None, scale=1.0, stream=None):
    """Next-token losses and the logits' gradient: logits [..., vocab] fp32 or
    bf16; targets [...] uint8, int32 or int64 (outside the vocabulary: ignored);
    weight [...] fp32 (0: ignored). loss [...] fp32 = -weight log softmax at the
    target; dlogits (None: not wanted; it may be logits) = scale * the gradient
    of the losses' sum. Returns (loss, dlogits)."""
    if stream is None:
        rc = (_fast or _native()).cross_entropy(logits, targets, loss, dlogits, weight, scale)
        if rc >= 0:
            _check(rc, "mb_cross_entropy")
            return loss, dlogits
    tt = _token_type(targets, "targets")
    if logits.dtype not in _DTYPES:
        raise TypeError(f"logits: unsupported dtype {logits.dtype}")
    rows, vocab = tuple(logits.shape[:-1]), logits.shape[-1]
    dev = logits.device
    _need(logits, "logits")
    _need(targets, "targets", None, rows, dev)
    _need(weight, "weight", torch.float32, rows, dev)
    _need(loss, "loss", torch.float32, rows, dev)
    _need(dlogits, "dlogits", logits.dtype, tuple(logits.shape), dev)
    rc = load_library().mb_cross_entropy(_ptr(logits), _DTYPES[logits.dtype], _ptr(targets), tt, _ptr(weight),
                                         float(scale), _ptr(loss), _ptr(dlogits), targets.numel(), vocab,
                                         _stream(stream, dev))
    _check(rc, "mb_cross_entropy")
    return loss, dlogits


class TensorList:
    """A list of tensors as the C ABI takes it, checked once; keeps them alive."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.array = (mb_tensor * len(self.tensors))()
        dev = getattr(self.tensors[0], "device", None) if self.tensors else None
        for a, t in zip(self.array, self.tensors):
            _need(t, "tensor", None, None, dev)
            if t.dtype not in _DTYPES:
                raise TypeError(f"unsupported dtype {t.dtype}")
            a.data, a.numel, a.dtype = t.data_ptr(), t.numel(), _DTYPES[t.dtype]
        self.address = ctypes.addressof(self.array)

    def __len__(self):
        return len(self.tensors)


def mb_tensor_list(tensors) -> TensorList:
    """The handle that mb_grad_norm and mb_grad_clip take, for tensors that stay where they are."""
    return TensorList(tensors)


def _tensor_list(tensors) -> TensorList:
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def mb_grad_norm_workspace_size() -> int:
    return int(load_library().mb_grad_norm_workspace_size())


def mb_grad_norm(tensors, norm=None, *, ws=None, stream=None):
    """norm [1] fp32 = the 2-norm over every element of `tensors` (an
    mb_tensor_list, or tensors: contiguous, fp32 or bf16, on one device)."""
    if type(tensors) is TensorList and len(tensors) and norm is not None and ws is not None and stream is None:
        rc = (_fast or _native()).grad_norm(tensors.address, len(tensors), tensors.tensors[0], norm, ws)
        if rc >= 0:
            _check(rc, "mb_grad_norm")
            return norm
    lst = _tensor_list(tensors)
    dev = lst.tensors[0].device if len(lst) else norm.device if norm is not None else torch.device("cuda")
    if norm is None:
        norm = torch.empty(1, device=dev)
    _need(norm, "norm", torch.float32, (1,), dev)
    if ws is None:
        ws = torch.zeros(mb_grad_norm_workspace_size(), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8, None, dev)
    rc = load_library().mb_grad_norm(lst.array, len(lst), _ptr(norm), _ptr(ws), ws.numel(), _stream(stream, dev))
    _check(rc, "mb_grad_norm")
    return norm


def mb_grad_clip(tensors, norm, max_norm, *, out=None, stream=None):
    """Scale `tensors` by max_norm / norm where max_norm < norm < inf (norm [1]
    on the device, from mb_grad_norm), in place or into `out` (as many tensors
    of the same sizes, fp32 or bf16 each; copied where nothing is clipped)."""
    if type(tensors) is TensorList and len(tensors) and stream is None and (
            out is None or type(out) is TensorList and len(out) == len(tensors)):
        rc = (_fast or _native()).grad_clip(tensors.address, len(tensors), tensors.tensors[0], norm, max_norm,
                                            0 if out is None else out.address, None if out is None else out.tensors[0])
        if rc >= 0:
            _check(rc, "mb_grad_clip")
            return tensors if out is None else out
    lst = _tensor_list(tensors)
    o = None if out is None else _tensor_list(out)
    if o is not None and len(o) != len(lst):
        raise ValueError(f"out has {len(o)} tensors, expected {len(lst)}")
    for t in () if not len(lst) else (norm, *(o.tensors[:1] if o is not None else ())):
        if t.device != lst.tensors[0].device:
            raise ValueError(f"tensor on {t.device}, expected {lst.tensors[0].device}")
    _need(norm, "norm", torch.float32, (1,))
    rc = load_library().mb_grad_clip(lst.array, None if o is None else o.array, len(lst), _ptr(norm), float(max_norm),
                                     _stream(stream, norm.device))
    _check(rc, "mb_grad_clip")
    return tensors if out is None else out


Q8_BLOCK = 128   # columns (and, of weights, rows) that share a scale of an 8-bit matrix


def mb_q8_scale_stride(width: int) -> int:
    """Bytes of scales of a row of an 8-bit matrix (0: width not accepted)."""
    return int(load_library().mb_q8_scale_stride(width))


def _here(dev):
    """The new calls launch on a stream of the current device: their tensors are there."""
    if dev.type == "cuda" and dev.index != torch.cuda.current_device():
        raise ValueError(f"tensors on {dev}, the current device is cuda:{torch.cuda.current_device()}")


def _need_q8(q, scales, name, block_rows, dev=None):
    """Checks an 8-bit matrix: q [rows, width] (torch.float8_e4m3fn, or uint8 holding it) and its scales."""
    for n, t in ((name, q), (name + "_scales", scales)):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{n} must be a torch.Tensor")
    if q.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise TypeError(f"{name}: dtype {q.dtype}, expected torch.float8_e4m3fn or torch.uint8")
    if q.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(q.shape)}, expected [rows, width]")
    _need(q, name, None, None, dev)
    rows, width = q.shape
    if width % 16 == 0:   # else the library refuses
        _need(scales, name + "_scales", torch.uint8, (-(-rows // block_rows), 4 * -(-width // (4 * Q8_BLOCK))), q.device)
    return rows, width


def _block_rows(block_rows):
    if block_rows not in (1, Q8_BLOCK):
        raise ValueError(f"block_rows {block_rows}, expected 1 or {Q8_BLOCK}")
    return int(block_rows)


def mb_rmsnorm_q8(residual, w, q, scales, *, add=None, eps=1e-5, stream=None):
    """residual [rows, width] fp32 (+= add), then its RMS norm times w [width]
    fp32 in 8 bits: q [rows, width] (torch.float8_e4m3fn, or uint8) and scales
    [rows, mb_q8_scale_stride(width)] uint8, one for 128 columns. add [rows,
    width] fp32 or bf16."""
    if stream is None:
        rc = (_fast or _native()).rmsnorm_q8(residual, w, q, scales, add, eps)
        if rc >= 0:
            _check(rc, "mb_rmsnorm_q8")
            return q, scales
    dev = residual.device
    rows, width = _need_q8(q, scales, "q", 1, dev)
    _need(residual, "residual", torch.float32, (rows, width), dev)
    _need(w, "w", torch.float32, (width,), dev)
    if add is not None and add.dtype not in _DTYPES:
        raise TypeError(f"add: unsupported dtype {add.dtype}")
    _need(add, "add", None, (rows, width), dev)
    _here(dev)
    dt = MB_BF16 if add is None else _DTYPES[add.dtype]
    rc = load_library().mb_rmsnorm_q8(_ptr(add), dt, _ptr(residual), _ptr(w), float(eps), _ptr(q), _ptr(scales), rows, width,
                                      _stream(stream, dev))
    _check(rc, "mb_rmsnorm_q8")
    return q, scales


def mb_quantize_q8(x, q, scales, *, block_rows=1, stream=None):
    """x [rows, width] fp32 or bf16 (contiguous or a column block of wider rows)
    in 8 bits: q [rows, width] (torch.float8_e4m3fn, or uint8), scales
    [ceil(rows / block_rows), mb_q8_scale_stride(width)] uint8, one for 128
    columns of block_rows rows: 1 (activations) or 128 (weights)."""
    if stream is None:
        rc = (_fast or _native()).quantize_q8(x, q, scales, block_rows)
        if rc >= 0:
            _check(rc, "mb_quantize_q8")
            return q, scales
    block_rows = _block_rows(block_rows)
    rows, width = _need_q8(q, scales, "q", block_rows)
    dev = q.device
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    if x.dtype not in _DTYPES:
        raise TypeError(f"x: unsupported dtype {x.dtype}")
    if tuple(x.shape) != (rows, width) or x.device != dev:
        raise ValueError(f"x: {tuple(x.shape)} on {x.device}, expected {(rows, width)} on {dev}")
    S = width if x.is_contiguous() or rows == 1 and x.stride(1) == 1 else x.stride(0)
    if not x.is_contiguous() and x.stride(1) != 1 or S < width:
        raise ValueError("x must be contiguous or a column block of wider rows")
    _here(dev)
    rc = load_library().mb_quantize_q8(_ptr(x), _DTYPES[x.dtype], S, block_rows, _ptr(q), _ptr(scales), rows, width,
                                       _stream(stream, dev))
    _check(rc, "mb_quantize_q8")
    return q, scales


def mb_dequantize_q8(q, scales, out, *, block_rows=1, stream=None):
    """The values that q and scales stand for: out [rows, width] fp32 or bf16."""
    if stream is None:
        rc = (_fast or _native()).dequantize_q8(q, scales, out, block_rows)
        if rc >= 0:
            _check(rc, "mb_dequantize_q8")
            return out
    block_rows = _block_rows(block_rows)
    rows, width = _need_q8(q, scales, "q", block_rows)
    if out.dtype not in _DTYPES:
        raise TypeError(f"out: unsupported dtype {out.dtype}")
    _need(out, "out", None, (rows, width), q.device)
    _here(q.device)
    rc = load_library().mb_dequantize_q8(_ptr(q), _ptr(scales), block_rows, _ptr(out), _DTYPES[out.dtype], rows, width,
                                         _stream(stream, q.device))
    _check(rc, "mb_dequantize_q8")
    return out


def mb_matmul_q8(a, a_scales, w, w_scales, out, *, ws=None, stream=None):
    """out = A W^T of 8-bit matrices: a [rows, width] with a_scales (block_rows
    1), w [n_out, width] with w_scales (block_rows 128). out fp32 or bf16:
    [rows, n_out], or [parts, rows, n_out / parts] for the product's columns in
    that many groups. ws: a workspace of 256 bytes (a wait that timed out is
    recorded there) or None."""
    if stream is None:
        rc = (_fast or _native()).matmul_q8(a, a_scales, w, w_scales, out, ws)
        if rc >= 0:
            _check(rc, "mb_matmul_q8")
            return out
    rows, width = _need_q8(a, a_scales, "a", 1)
    dev = a.device
    n_out, k = _need_q8(w, w_scales, "w", Q8_BLOCK, dev)
    if k != width:
        raise ValueError(f"w: rows of {k}, expected {width}")
    if out.dtype not in _DTYPES:
        raise TypeError(f"out: unsupported dtype {out.dtype}")
    part = out.shape[-1]
    parts = out.shape[0] if out.dim() == 3 else 1
    _need(out, "out", None, (rows, n_out) if out.dim() == 2 else (parts, rows, part), dev)
    if parts * part != n_out:
        raise ValueError(f"out: {parts} groups of {part} columns, expected {n_out} in all")
    _need(ws, "ws", torch.uint8, None, dev)
    _here(dev)
    rc = load_library().mb_matmul_q8(_ptr(a), _ptr(a_scales), _ptr(w), _ptr(w_scales), _ptr(out), _DTYPES[out.dtype], rows,
                                     n_out, width, part, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream, dev))
    _check(rc, "mb_matmul_q8")
    return out


def mb_matmul_q8_form(rows, n_out, width, dtype=torch.bfloat16):
    """How mb_matmul_q8 takes a product of these sizes on the current device:
    {"pair", "parts", "height", "deep", "tiles"} (2 where pairs of CTAs share
    tiles; parts of each sum; rows of a tile; 128-column blocks fetched at a
    time; tiles to a CTA)."""
    if dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {dtype}")
    form = (ctypes.c_int64 * 5)()
    _check(load_library().mb_matmul_q8_form(int(rows), int(n_out), int(width), _DTYPES[dtype], form), "mb_matmul_q8_form")
    return dict(zip(("pair", "parts", "height", "deep", "tiles"), form))


def mb_sample(logits, u, tokens=None, *, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, stream=None):
    """Draw a token of every row of logits [n, vocab] (fp32 or bf16) by the
    random numbers u [n] fp32 in [0, 1): temperature, then the top_k likeliest
    tokens, of these the nucleus of mass top_p, of these those at least min_p
    times as likely as the likeliest; each [n] (fp32; top_k int32) or None.
    tokens [n] int32 or int64 (None: a new int64 tensor): -1 where every token
    is masked (-inf). prob [n] fp32 (if given): what the token was drawn with."""
    if tokens is not None and stream is None:
        rc = (_fast or _native()).sample(logits, u, tokens, temperature, top_k, top_p, min_p, prob)
        if rc >= 0:
            _check(rc, "mb_sample")
            return tokens
    if logits.dtype not in _DTYPES:
        raise TypeError(f"logits: unsupported dtype {logits.dtype}")
    n, vocab = logits.shape
    dev = logits.device
    _need(logits, "logits")
    if tokens is None:
        tokens = torch.empty(n, dtype=torch.int64, device=dev)
    if tokens.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"tokens: dtype {tokens.dtype}, expected torch.int32 or torch.int64")
    _need(tokens, "tokens", None, (n,), dev)
    for name, t, dtype in (("u", u, torch.float32), ("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                           ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32), ("prob", prob, torch.float32)):
        _need(t, name, dtype, (n,), dev)
    if u is None:
        raise TypeError("u must be a torch.Tensor")
    _here(dev)
    rc = load_library().mb_sample(_ptr(logits), _DTYPES[logits.dtype], _ptr(u), _ptr(temperature), _ptr(top_k), _ptr(top_p),
                                  _ptr(min_p), _ptr(tokens), _TOKENS[tokens.dtype], _ptr(prob), n, vocab, _stream(stream, dev))
    _check(rc, "mb_sample")
    return tokens


def mb_selftest_timeout(ws, wait_cycles, stream=None):
    """Run the bounded-wait diagnostic: one of four warps waits wait_cycles SM
    clocks on a barrier nothing arrives on, all four give up, and
    MB_ERR_TIMEOUT is recorded in ws (read it with mb_check)."""
    _need(ws, "ws", torch.uint8)
    rc = load_library().mb_selftest_timeout(_ptr(ws), ws.numel(), int(wait_cycles), _stream(stream, ws.device))
    _check(rc, "mb_selftest_timeout")


def mb_check(ws, stream=None):
    """Read and clear the workspace status block: (status, detail)."""
    detail = ctypes.c_int64(-1)
    dev = torch.device("cuda") if ws is None else ws.device   # no workspace: the library's answer
    rc = load_library().mb_check(_ptr(ws), _stream(stream, dev), ctypes.byref(detail))
    return int(rc), int(detail.value)

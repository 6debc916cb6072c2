"""Binding for the log-probability entry points of libmi355conv.so: the same names as include/mi355lp.h, marshalling only
(every compute step runs in the HIP kernels; see binding.py for the extension that the compute calls go through)."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as _b

_ready = False

DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.float64: 3}  # mi355_dtype_t


@dataclass(frozen=True)
class LpParams:
    """Mirror of lp_params_t; dtype is torch's."""
    rows: int
    vocab: int
    dtype: torch.dtype = torch.float32
    top: int = 0
    entropy: int = 1
    scale: float = 1.0


class _CParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("rows", "vocab", "dtype", "top", "entropy")] + [("scale", ctypes.c_float)]


def _load():
    global _ready
    lib = _b._load()
    if not _ready:
        vp, sz, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
        lib.lp_desc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_CParams)]
        lib.lp_desc_destroy.argtypes = [vp]
        lib.lp_desc_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.lp_desc_kernel_names.argtypes = [vp]
        lib.lp_desc_kernel_names.restype = ctypes.c_char_p
        lib.lp_forward.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.lp_backward.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, i64, vp]
        lib.lp_forward_backward.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
        for name in ("lp_desc_create", "lp_desc_destroy", "lp_desc_workspace_bytes", "lp_forward", "lp_backward",
                     "lp_forward_backward"):
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


def _dtype(dtype, allowed) -> int:
    code = DTYPES.get(dtype)
    if code is None or code not in allowed:
        raise TypeError(f"dtype: {dtype} is not among those of this operator")
    return code


def _fits(value, bits, where) -> int:
    """An integer for a C field of so many bits: ctypes would take its lowest ones."""
    value = int(value)
    if not -1 << bits - 1 <= value < 1 << bits - 1:
        raise _b.ConvError(_b.CONV_ESHAPE if value > 0 else _b.CONV_EINVAL, where)
    return value


class LpDesc:
    """Owner of an lp_desc_t*; destroyed with the Python object (or lp_desc_destroy)."""

    def __init__(self, handle: int, params: LpParams):
        self.handle = handle
        self.params = params
        self._plan = None

    def __del__(self):
        try:
            lp_desc_destroy(self)
        except Exception:
            pass


def lp_desc_create(params: LpParams) -> LpDesc:
    fits = lambda value: _fits(value, 32, "lp_desc_create")
    c = _CParams(fits(params.rows), fits(params.vocab), _dtype(params.dtype, (0, 1, 2)), fits(params.top), fits(params.entropy),
                 float(params.scale))
    out = ctypes.c_void_p()
    _b._check(_load().lp_desc_create(ctypes.byref(out), ctypes.byref(c)), "lp_desc_create")
    desc = LpDesc(out.value, params)
    desc._plan = _b._marshal.lp_plan(desc.handle, c.rows, c.vocab, c.dtype, c.top)
    return desc


def lp_desc_destroy(desc: LpDesc) -> None:
    if desc.handle:
        desc._plan = None
        _load().lp_desc_destroy(desc.handle)
        desc.handle = None


def lp_desc_workspace_bytes(desc: LpDesc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().lp_desc_workspace_bytes(desc.handle, ctypes.byref(b)), "lp_desc_workspace_bytes")
    return int(b.value)


def lp_desc_kernel_names(desc: LpDesc) -> str:
    return _load().lp_desc_kernel_names(desc.handle).decode()


def _rows(t, params, name):
    """Address and row stride of a blob whose rows are dense but may lie apart."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA/HIP tensor (there is no CPU path)")
    if t.dtype != params.dtype:
        raise TypeError(f"{name}: expected a {params.dtype} tensor")
    if tuple(t.shape) != (params.rows, params.vocab):
        raise ValueError(f"{name}: expected shape {(params.rows, params.vocab)}, got {tuple(t.shape)}")
    if (params.vocab > 1 and t.stride(1) != 1) or (params.rows > 1 and t.stride(0) < params.vocab):
        raise TypeError(f"{name}: expected dense rows that do not overlap")
    return t.data_ptr() or None, t.stride(0) if params.rows > 1 else params.vocab


def lp_forward(desc, logits, token, logp, entropy=None, stats=None, top_logp=None, top_token=None, ws=None, stream=None) -> None:
    status = _b._marshal.lp_forward(desc._plan, logits, token, logp, entropy, stats, top_logp, top_token, ws, stream)
    if status is not None:
        return _b._check(status, "lp_forward")
    p, i32 = desc.params, torch.int32
    x, stride = _rows(logits, p, "logits")
    wp, wb = _b._ws(ws)
    _b._check(_load().lp_forward(desc.handle, x, stride, _b._ptr(token, (p.rows,), "token", i32), _b._ptr(logp, (p.rows,), "logp"),
                                 _b._ptr(entropy, (p.rows,), "entropy"), _b._ptr(stats, (p.rows, 4), "stats"),
                                 _b._ptr(top_logp, (p.rows, p.top), "top_logp"), _b._ptr(top_token, (p.rows, p.top), "top_token", i32),
                                 wp, wb, _b._stream(stream)), "lp_forward")


def lp_backward(desc, logits, token, stats, d_logp, d_entropy, d_logits, stream=None) -> None:
    status = _b._marshal.lp_backward(desc._plan, logits, token, stats, d_logp, d_entropy, d_logits, stream)
    if status is not None:
        return _b._check(status, "lp_backward")
    p = desc.params
    x, stride = _rows(logits, p, "logits")
    g, d_stride = _rows(d_logits, p, "d_logits")
    _b._check(_load().lp_backward(desc.handle, x, stride, _b._ptr(token, (p.rows,), "token", torch.int32),
                                  _b._ptr(stats, (p.rows, 4), "stats"), _b._ptr(d_logp, (p.rows,), "d_logp"),
                                  _b._ptr(d_entropy, (p.rows,), "d_entropy"), g, d_stride, _b._stream(stream)), "lp_backward")


def lp_forward_backward(desc, logits, token, d_logp, d_entropy, logp, entropy, d_logits, ws=None, stream=None) -> None:
    status = _b._marshal.lp_forward_backward(desc._plan, logits, token, d_logp, d_entropy, logp, entropy, d_logits, ws, stream)
    if status is not None:
        return _b._check(status, "lp_forward_backward")
    p = desc.params
    x, stride = _rows(logits, p, "logits")
    g, d_stride = _rows(d_logits, p, "d_logits")
    wp, wb = _b._ws(ws)
    _b._check(_load().lp_forward_backward(desc.handle, x, stride, _b._ptr(token, (p.rows,), "token", torch.int32),
                                          _b._ptr(d_logp, (p.rows,), "d_logp"), _b._ptr(d_entropy, (p.rows,), "d_entropy"),
                                          _b._ptr(logp, (p.rows,), "logp"), _b._ptr(entropy, (p.rows,), "entropy"), g, d_stride,
                                          wp, wb, _b._stream(stream)), "lp_forward_backward")

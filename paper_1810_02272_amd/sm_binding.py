"""Binding for the token-drawing entry points of libmi355conv.so: the same names as include/mi355sm.h, marshalling only
(every compute step runs in the HIP kernels; see binding.py for the extension that the compute calls go through)."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as _b
from .lp_binding import _dtype, _fits, _rows

_ready = False


@dataclass(frozen=True)
class SmParams:
    """Mirror of sm_params_t; dtype is torch's."""
    rows: int
    vocab: int
    dtype: torch.dtype = torch.float32


class _CParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("rows", "vocab", "dtype")]


def _load():
    global _ready
    lib = _b._load()
    if not _ready:
        vp, sz, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
        lib.sm_desc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_CParams)]
        lib.sm_desc_destroy.argtypes = [vp]
        lib.sm_desc_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.sm_desc_kernel_names.argtypes = [vp]
        lib.sm_desc_kernel_names.restype = ctypes.c_char_p
        lib.sm_sample.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        for name in ("sm_desc_create", "sm_desc_destroy", "sm_desc_workspace_bytes", "sm_sample"):
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


class SmDesc:
    """Owner of an sm_desc_t*; destroyed with the Python object (or sm_desc_destroy)."""

    def __init__(self, handle: int, params: SmParams):
        self.handle = handle
        self.params = params
        self._plan = None

    def __del__(self):
        try:
            sm_desc_destroy(self)
        except Exception:
            pass


def sm_desc_create(params: SmParams) -> SmDesc:
    fits = lambda value: _fits(value, 32, "sm_desc_create")
    c = _CParams(fits(params.rows), fits(params.vocab), _dtype(params.dtype, (0, 1, 2)))
    out = ctypes.c_void_p()
    _b._check(_load().sm_desc_create(ctypes.byref(out), ctypes.byref(c)), "sm_desc_create")
    desc = SmDesc(out.value, params)
    desc._plan = _b._marshal.sm_plan(desc.handle, c.rows, c.vocab, c.dtype)
    return desc


def sm_desc_destroy(desc: SmDesc) -> None:
    if desc.handle:
        desc._plan = None
        _load().sm_desc_destroy(desc.handle)
        desc.handle = None


def sm_desc_workspace_bytes(desc: SmDesc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().sm_desc_workspace_bytes(desc.handle, ctypes.byref(b)), "sm_desc_workspace_bytes")
    return int(b.value)


def sm_desc_kernel_names(desc: SmDesc) -> str:
    return _load().sm_desc_kernel_names(desc.handle).decode()


def sm_sample(desc, logits, u, scale, top_k, top_p, min_p, token, logp=None, ws=None, stream=None) -> None:
    status = _b._marshal.sm_sample(desc._plan, logits, u, scale, top_k, top_p, min_p, token, logp, ws, stream)
    if status is not None:
        return _b._check(status, "sm_sample")
    p, i32 = desc.params, torch.int32
    x, stride = _rows(logits, p, "logits")
    row = lambda t, name, dtype=torch.float32: _b._ptr(t, (p.rows,), name, dtype)
    wp, wb = _b._ws(ws)
    _b._check(_load().sm_sample(desc.handle, x, stride, row(u, "u"), row(scale, "scale"), row(top_k, "top_k", i32), row(top_p, "top_p"),
                                row(min_p, "min_p"), row(token, "token", i32), row(logp, "logp"), wp, wb, _b._stream(stream)), "sm_sample")

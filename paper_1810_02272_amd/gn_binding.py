"""Binding for the gradient-norm entry points of libmi355conv.so: the same names as include/mi355gn.h, marshalling only
(every compute step runs in the HIP kernels; see binding.py for the extension that the compute calls go through)."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as _b
from .lp_binding import DTYPES, _fits

_ready = False


@dataclass(frozen=True)
class GnParams:
    """Mirror of gn_params_t: for each tensor its number of elements and its type (torch's)."""
    counts: tuple
    dtypes: tuple

    def __post_init__(self):
        object.__setattr__(self, "counts", tuple(map(int, self.counts)))
        object.__setattr__(self, "dtypes", tuple(self.dtypes))
        if len(self.counts) != len(self.dtypes):
            raise ValueError("one type for each count")


class _CParams(ctypes.Structure):
    _fields_ = [("tensors", ctypes.c_int32), ("counts", ctypes.POINTER(ctypes.c_int64)), ("dtypes", ctypes.POINTER(ctypes.c_int32))]


def _load():
    global _ready
    lib = _b._load()
    if not _ready:
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        lib.gn_desc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_CParams)]
        lib.gn_desc_destroy.argtypes = [vp]
        lib.gn_desc_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.gn_desc_kernel_names.argtypes = [vp]
        lib.gn_desc_kernel_names.restype = ctypes.c_char_p
        lib.gn_clip.argtypes = [vp, vp, ctypes.c_double, vp, vp, vp, sz, vp]
        for name in ("gn_desc_create", "gn_desc_destroy", "gn_desc_workspace_bytes", "gn_clip"):
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


class GnDesc:
    """Owner of a gn_desc_t*; destroyed with the Python object (or gn_desc_destroy)."""

    def __init__(self, handle: int, params: GnParams):
        self.handle = handle
        self.params = params
        self._plan = None

    def __del__(self):
        try:
            gn_desc_destroy(self)
        except Exception:
            pass


def gn_desc_create(params: GnParams) -> GnDesc:
    n = len(params.counts)
    codes = list(map(DTYPES.get, params.dtypes))
    if None in codes:
        raise TypeError(f"dtypes: {params.dtypes[codes.index(None)]} is not among those of this operator")
    counts = [_fits(count, 64, "gn_desc_create") for count in params.counts]
    c = _CParams(n, (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*codes))
    out = ctypes.c_void_p()
    _b._check(_load().gn_desc_create(ctypes.byref(out), ctypes.byref(c)), "gn_desc_create")
    desc = GnDesc(out.value, params)
    desc._plan = _b._marshal.gn_plan(desc.handle, params.counts, tuple(codes))
    return desc


def gn_desc_destroy(desc: GnDesc) -> None:
    if desc.handle:
        desc._plan = None
        _load().gn_desc_destroy(desc.handle)
        desc.handle = None


def gn_desc_workspace_bytes(desc: GnDesc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().gn_desc_workspace_bytes(desc.handle, ctypes.byref(b)), "gn_desc_workspace_bytes")
    return int(b.value)


def gn_desc_kernel_names(desc: GnDesc) -> str:
    return _load().gn_desc_kernel_names(desc.handle).decode()


def _pointers(tensors, params, name):
    tensors = list(tensors)
    if len(tensors) != len(params.counts):
        raise ValueError(f"{name}: expected {len(params.counts)} tensors, got {len(tensors)}")
    out = (ctypes.c_void_p * max(len(tensors), 1))()
    for i, (t, count, dtype) in enumerate(zip(tensors, params.counts, params.dtypes)):
        out[i] = _b._ptr(t, None, f"{name}[{i}]", dtype)
        if t is not None and t.numel() != count:
            raise ValueError(f"{name}[{i}]: expected {count} elements, got {t.numel()}")
    return out


def gn_clip(desc, grads, limit, outs=None, norm=None, ws=None, stream=None) -> None:
    """outs=None: in place."""
    if not isinstance(grads, (list, tuple)):
        grads = list(grads)  # an iterator is read once, also where the outputs are the gradients
    if outs is None:
        outs = grads
    status = _b._marshal.gn_clip(desc._plan, grads, limit, outs, norm, ws, stream)
    if status is not None:
        return _b._check(status, "gn_clip")
    wp, wb = _b._ws(ws)
    _b._check(_load().gn_clip(desc.handle, _pointers(grads, desc.params, "grads"), float(limit),
                              _pointers(outs, desc.params, "outs"), _b._ptr(norm, (1,), "norm"), wp, wb, _b._stream(stream)),
              "gn_clip")

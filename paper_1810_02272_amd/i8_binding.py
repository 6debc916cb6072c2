"""Binding for the entry points of libmi355conv.so on 8-bit integers: the same names as include/mi355i8.h, marshalling only
(every compute step runs in the HIP kernels; see binding.py for the extension that the compute calls go through)."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as _b
from .lp_binding import _dtype, _fits

_ready = False


@dataclass(frozen=True)
class I8Params:
    """Mirror of i8_params_t; dtype is torch's."""
    m: int
    k: int
    num_output: int
    dtype: torch.dtype = torch.bfloat16
    bias_term: int = 0
    relu: int = 0


class _CParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("m", "k", "num_output", "dtype", "bias_term", "relu")]


def _load():
    global _ready
    lib = _b._load()
    if not _ready:
        vp, sz, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
        lib.i8_desc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_CParams)]
        lib.i8_desc_destroy.argtypes = [vp]
        lib.i8_desc_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.i8_desc_row_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.i8_desc_kernel_names.argtypes = [vp]
        lib.i8_desc_kernel_names.restype = ctypes.c_char_p
        lib.i8_pack.argtypes = [vp] * 5
        lib.i8_quantise.argtypes = [vp] * 5
        lib.i8_forward.argtypes = [vp] * 9 + [sz, vp]
        lib.i8_backward_filter.argtypes = [vp] * 6 + [f32, vp, sz, vp]
        lib.i8_backward_data.argtypes = [vp] * 6 + [sz, vp]
        for name in ("i8_desc_create", "i8_desc_destroy", "i8_desc_workspace_bytes", "i8_desc_row_bytes", "i8_pack", "i8_quantise",
                     "i8_forward", "i8_backward_filter", "i8_backward_data"):
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


class I8Desc:
    """Owner of an i8_desc_t*; destroyed with the Python object (or i8_desc_destroy)."""

    def __init__(self, handle: int, params: I8Params):
        self.handle = handle
        self.params = params
        self.row = 0
        self._plan = None

    def __del__(self):
        try:
            i8_desc_destroy(self)
        except Exception:
            pass


def i8_desc_create(params: I8Params) -> I8Desc:
    p = params
    fits = lambda value: _fits(value, 32, "i8_desc_create")
    c = _CParams(fits(p.m), fits(p.k), fits(p.num_output), _dtype(p.dtype, (0, 1, 2)), fits(p.bias_term), fits(p.relu))
    out = ctypes.c_void_p()
    _b._check(_load().i8_desc_create(ctypes.byref(out), ctypes.byref(c)), "i8_desc_create")
    desc = I8Desc(out.value, params)
    desc.row = i8_desc_row_bytes(desc)
    desc._plan = _b._marshal.i8_plan(desc.handle, c.m, c.k, c.num_output, c.dtype, desc.row)
    return desc


def i8_desc_destroy(desc: I8Desc) -> None:
    if desc.handle:
        desc._plan = None
        _load().i8_desc_destroy(desc.handle)
        desc.handle = None


def i8_desc_workspace_bytes(desc: I8Desc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().i8_desc_workspace_bytes(desc.handle, ctypes.byref(b)), "i8_desc_workspace_bytes")
    return int(b.value)


def i8_desc_row_bytes(desc: I8Desc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().i8_desc_row_bytes(desc.handle, ctypes.byref(b)), "i8_desc_row_bytes")
    return int(b.value)


def i8_desc_kernel_names(desc: I8Desc) -> str:
    return _load().i8_desc_kernel_names(desc.handle).decode()


def _weights(desc, w_codes, w_scale):
    return (_b._ptr(w_codes, (desc.params.num_output, desc.row), "w_codes", torch.int8),
            _b._ptr(w_scale, (desc.params.num_output,), "w_scale"))


def _kept(desc, codes, scale):
    return _b._ptr(codes, (desc.params.m, desc.row), "codes", torch.int8), _b._ptr(scale, (desc.params.m,), "scale")


def i8_pack(desc, w, w_codes, w_scale, stream=None) -> None:
    p = desc.params
    _b._check(_load().i8_pack(desc.handle, _b._ptr(w, (p.num_output, p.k), "w", p.dtype), *_weights(desc, w_codes, w_scale),
                              _b._stream(stream)), "i8_pack")


def i8_quantise(desc, x, codes, scale, stream=None) -> None:
    status = _b._marshal.i8_quantise(desc._plan, x, codes, scale, stream)
    if status is not None:
        return _b._check(status, "i8_quantise")
    p = desc.params
    _b._check(_load().i8_quantise(desc.handle, _b._ptr(x, (p.m, p.k), "x", p.dtype), *_kept(desc, codes, scale), _b._stream(stream)),
              "i8_quantise")


def i8_forward(desc, x, w_codes, w_scale, bias, y, codes, scale, ws=None, stream=None) -> None:
    status = _b._marshal.i8_forward(desc._plan, x, w_codes, w_scale, bias, y, codes, scale, ws, stream)
    if status is not None:
        return _b._check(status, "i8_forward")
    p = desc.params
    wp, wb = _b._ws(ws)
    _b._check(_load().i8_forward(desc.handle, _b._ptr(x, (p.m, p.k), "x", p.dtype), *_weights(desc, w_codes, w_scale),
                                 _b._ptr(bias, (p.num_output,), "bias", p.dtype), _b._ptr(y, (p.m, p.num_output), "y", p.dtype),
                                 *_kept(desc, codes, scale), wp, wb, _b._stream(stream)), "i8_forward")


def i8_backward_filter(desc, codes, scale, dz, dw, db=None, beta=0.0, ws=None, stream=None) -> None:
    status = _b._marshal.i8_backward_filter(desc._plan, codes, scale, dz, dw, db, beta, ws, stream)
    if status is not None:
        return _b._check(status, "i8_backward_filter")
    p = desc.params
    wp, wb = _b._ws(ws)
    _b._check(_load().i8_backward_filter(desc.handle, *_kept(desc, codes, scale), _b._ptr(dz, (p.m, p.num_output), "dz", p.dtype),
                                         _b._ptr(dw, (p.num_output, p.k), "dw"), _b._ptr(db, (p.num_output,), "db"), beta, wp, wb,
                                         _b._stream(stream)), "i8_backward_filter")


def i8_backward_data(desc, w_codes, w_scale, dz, dx, ws=None, stream=None) -> None:
    status = _b._marshal.i8_backward_data(desc._plan, w_codes, w_scale, dz, dx, ws, stream)
    if status is not None:
        return _b._check(status, "i8_backward_data")
    p = desc.params
    wp, wb = _b._ws(ws)
    _b._check(_load().i8_backward_data(desc.handle, *_weights(desc, w_codes, w_scale), _b._ptr(dz, (p.m, p.num_output), "dz", p.dtype),
                                       _b._ptr(dx, (p.m, p.k), "dx", p.dtype), wp, wb, _b._stream(stream)), "i8_backward_data")

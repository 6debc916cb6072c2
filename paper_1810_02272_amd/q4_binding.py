"""Binding for the entry points of libmi355conv.so on 4-bit weights: the same names as include/mi355q4.h, marshalling only
(every compute step runs in the HIP kernels; see binding.py for the extension that the compute calls go through)."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as _b
from .lp_binding import _dtype, _fits

_ready = False


@dataclass(frozen=True)
class Q4Params:
    """Mirror of q4_params_t; dtype is torch's."""
    m: int
    k: int
    num_output: int
    dtype: torch.dtype = torch.bfloat16
    group: int = 32
    bias_term: int = 0
    relu: int = 0


class _CParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("m", "k", "num_output", "dtype", "group", "bias_term", "relu")]


def _load():
    global _ready
    lib = _b._load()
    if not _ready:
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        lib.q4_desc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_CParams)]
        lib.q4_desc_destroy.argtypes = [vp]
        lib.q4_desc_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.q4_desc_packed_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        lib.q4_desc_kernel_names.argtypes = [vp]
        lib.q4_desc_kernel_names.restype = ctypes.c_char_p
        lib.q4_pack.argtypes = [vp, vp, vp, vp, vp]
        lib.q4_forward.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
        for name in ("q4_desc_create", "q4_desc_destroy", "q4_desc_workspace_bytes", "q4_desc_packed_bytes", "q4_pack",
                     "q4_forward"):
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


class Q4Desc:
    """Owner of a q4_desc_t*; destroyed with the Python object (or q4_desc_destroy)."""

    def __init__(self, handle: int, params: Q4Params):
        self.handle = handle
        self.params = params
        self._plan = None

    def __del__(self):
        try:
            q4_desc_destroy(self)
        except Exception:
            pass


def q4_desc_create(params: Q4Params) -> Q4Desc:
    p = params
    fits = lambda value: _fits(value, 32, "q4_desc_create")
    c = _CParams(fits(p.m), fits(p.k), fits(p.num_output), _dtype(p.dtype, (0, 1, 2)), fits(p.group), fits(p.bias_term), fits(p.relu))
    out = ctypes.c_void_p()
    _b._check(_load().q4_desc_create(ctypes.byref(out), ctypes.byref(c)), "q4_desc_create")
    desc = Q4Desc(out.value, params)
    desc._plan = _b._marshal.q4_plan(desc.handle, c.m, c.k, c.num_output, c.dtype, q4_desc_packed_bytes(desc))
    return desc


def q4_desc_destroy(desc: Q4Desc) -> None:
    if desc.handle:
        desc._plan = None
        _load().q4_desc_destroy(desc.handle)
        desc.handle = None


def q4_desc_workspace_bytes(desc: Q4Desc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().q4_desc_workspace_bytes(desc.handle, ctypes.byref(b)), "q4_desc_workspace_bytes")
    return int(b.value)


def q4_desc_packed_bytes(desc: Q4Desc) -> int:
    b = ctypes.c_size_t()
    _b._check(_load().q4_desc_packed_bytes(desc.handle, ctypes.byref(b)), "q4_desc_packed_bytes")
    return int(b.value)


def q4_desc_kernel_names(desc: Q4Desc) -> str:
    return _load().q4_desc_kernel_names(desc.handle).decode()


def q4_pack(desc, codes, scales, packed, stream=None) -> None:
    p = desc.params
    _b._check(_load().q4_pack(desc.handle, _b._ptr(codes, (p.num_output, (p.k + 1) // 2), "codes", torch.uint8),
                              _b._ptr(scales, (p.num_output, -(-p.k // p.group)), "scales", torch.bfloat16),
                              _b._ptr(packed, (q4_desc_packed_bytes(desc),), "packed", torch.uint8), _b._stream(stream)), "q4_pack")


def q4_forward(desc, x, packed, bias, y, ws=None, stream=None) -> None:
    status = _b._marshal.q4_forward(desc._plan, x, packed, bias, y, ws, stream)
    if status is not None:
        return _b._check(status, "q4_forward")
    p = desc.params
    wp, wb = _b._ws(ws)
    _b._check(_load().q4_forward(desc.handle, _b._ptr(x, (p.m, p.k), "x", p.dtype),
                                 _b._ptr(packed, (q4_desc_packed_bytes(desc),), "packed", torch.uint8),
                                 _b._ptr(bias, (p.num_output,), "bias", p.dtype), _b._ptr(y, (p.m, p.num_output), "y", p.dtype),
                                 wp, wb, _b._stream(stream)), "q4_forward")

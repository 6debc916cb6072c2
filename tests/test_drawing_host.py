"""Host side of drawing tokens and of layers in 8 bits, without a device: exported names, descriptors, refusals."""
import ctypes
import os
import re

import pytest
import torch

import paper_1810_02272_amd as lib
from paper_1810_02272_amd import binding, i8_binding, sm_binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64
f, odd = ctypes.c_void_p(256), ctypes.c_void_p(264)  # never dereferenced: every call below returns before any launch
EINVAL, ESHAPE, EWORKSPACE, OK = binding.CONV_EINVAL, binding.CONV_ESHAPE, binding.CONV_EWORKSPACE, binding.CONV_OK


@pytest.mark.parametrize("prefix,names", [
    ("sm", {"desc_create", "desc_destroy", "desc_workspace_bytes", "desc_kernel_names", "sample"}),
    ("i8", {"desc_create", "desc_destroy", "desc_workspace_bytes", "desc_row_bytes", "desc_kernel_names", "pack", "quantise", "forward",
            "backward_filter", "backward_data"})])
def test_every_declared_symbol_is_exported_and_bound(prefix, names):
    header = open(os.path.join(ROOT, "include", f"mi355{prefix}.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(rf"\b({prefix}_[a-z0-9_]+)\s*\(", header))
    assert declared == {f"{prefix}_{n}" for n in names}
    c = ctypes.CDLL(lib.library_path())
    for name in declared:
        assert hasattr(c, name) and hasattr(lib, name), name


# ---- drawing tokens ----

@pytest.mark.parametrize("bad,status", [(dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(vocab=-5), EINVAL), (dict(vocab=1 << 30), ESHAPE)])
def test_sm_parameters(bad, status):
    with pytest.raises(lib.ConvError) as e:
        lib.sm_desc_create(lib.SmParams(**{**dict(rows=4, vocab=100, dtype=F32), **bad}))
    assert e.value.status == status
    for dtype in (F64, torch.int32):
        with pytest.raises(TypeError):
            lib.sm_desc_create(lib.SmParams(4, 100, dtype))


def sample(c, handle, x=f, stride=100, u=f, limits=(f, f, f, f), token=f, logp=f, ws=f, ws_bytes=1 << 40):
    return c.sm_sample(handle, x, stride, u, *limits, token, logp, ws, ws_bytes, None)


def test_sm_calls():
    c = sm_binding._load()
    d = lib.sm_desc_create(lib.SmParams(4, 100, F32))
    none = lib.sm_desc_create(lib.SmParams(0, 100, F32))
    assert c.sm_desc_create(None, None) == EINVAL and c.sm_desc_destroy(None) == EINVAL and c.sm_desc_workspace_bytes(None, None) == EINVAL
    assert c.sm_desc_kernel_names(None) == b""
    assert sample(c, None) == EINVAL
    assert sample(c, d.handle, x=None) == EINVAL
    assert sample(c, d.handle, stride=99) == EINVAL  # rows overlap
    assert sample(c, d.handle, u=None) == EINVAL
    assert sample(c, d.handle, token=None) == EINVAL
    assert sample(c, none.handle, None, 0, None, (None,) * 4, None, None, None, 0) == OK
    for rows in (1, 3, 64, 300):
        for vocab in (100, 50257, 128256, 700000):
            large = lib.sm_desc_create(lib.SmParams(rows, vocab, BF16))
            if lib.sm_desc_workspace_bytes(large):
                assert sample(c, large.handle, stride=vocab, ws=None) == EWORKSPACE
                assert sample(c, large.handle, stride=vocab, ws_bytes=lib.sm_desc_workspace_bytes(large) - 1) == EWORKSPACE
                assert sample(c, large.handle, stride=vocab, ws=odd) == EINVAL


def test_sm_binding_refuses_what_is_not_on_the_device():
    d = lib.sm_desc_create(lib.SmParams(4, 100, F32))
    with pytest.raises(TypeError):
        lib.sm_sample(d, torch.zeros(4, 100), torch.zeros(4), None, None, None, None, torch.zeros(4, dtype=torch.int32))


# ---- layers in 8 bits ----

@pytest.mark.parametrize("bad,status", [(dict(m=-1), EINVAL), (dict(k=0), EINVAL), (dict(num_output=0), EINVAL), (dict(bias_term=2), EINVAL), (dict(relu=-1), EINVAL),
                                        (dict(k=133121), ESHAPE), (dict(m=1 << 25), ESHAPE), (dict(num_output=1 << 25), ESHAPE),
                                        (dict(m=1 << 15, k=8, num_output=1 << 15), ESHAPE)])
def test_i8_parameters(bad, status):
    with pytest.raises(lib.ConvError) as e:
        lib.i8_desc_create(lib.I8Params(**{**dict(m=2, k=64, num_output=8, dtype=BF16), **bad}))
    assert e.value.status == status
    with pytest.raises(TypeError):
        lib.i8_desc_create(lib.I8Params(2, 64, 8, F64))


def test_i8_calls():
    c = i8_binding._load()
    d = lib.i8_desc_create(lib.I8Params(2, 64, 8, BF16, 1, 0))
    plain = lib.i8_desc_create(lib.I8Params(2, 64, 8, BF16, 0, 0))
    none = lib.i8_desc_create(lib.I8Params(0, 64, 8, BF16, 1, 0))
    split = lib.i8_desc_create(lib.I8Params(4000, 64, 8, BF16, 1, 0))
    across = lib.i8_desc_create(lib.I8Params(8, 64, 4000, BF16, 1, 0))
    big = 1 << 40
    assert [lib.i8_desc_row_bytes(lib.i8_desc_create(lib.I8Params(1, k, 1))) for k in (1, 127, 128, 129, 133120)] == [128, 128, 128, 256, 133120]
    assert c.i8_desc_create(None, None) == EINVAL and c.i8_desc_destroy(None) == EINVAL
    assert c.i8_desc_row_bytes(None, None) == EINVAL and c.i8_desc_workspace_bytes(None, None) == EINVAL
    assert c.i8_desc_kernel_names(None) == b""
    for call, handle in ((c.i8_pack, d.handle), (c.i8_quantise, d.handle)):
        assert call(None, f, f, f, None) == EINVAL
        for args in ((None, f, f), (f, None, f), (f, f, None), (f, odd, f)):
            assert call(handle, *args, None) == EINVAL
    assert c.i8_quantise(none.handle, None, None, None, None) == OK
    # x, w_codes, w_scale, bias, y, codes, scale
    full = [f] * 7
    assert c.i8_forward(None, *full, f, big, None) == EINVAL
    for at in (1, 2, 3, 4, 5, 6):
        assert c.i8_forward(d.handle, *[None if i == at else f for i in range(7)], f, big, None) == EINVAL, at
    for at in (1, 5):
        assert c.i8_forward(d.handle, *[odd if i == at else f for i in range(7)], f, big, None) == EINVAL, at
    assert c.i8_forward(plain.handle, *full, f, big, None) == EINVAL  # bias unexpected
    assert c.i8_forward(none.handle, None, f, f, f, None, None, None, None, 0, None) == OK
    # codes, scale, dz, dw, db
    assert c.i8_backward_filter(None, f, f, f, f, f, 0.0, f, big, None) == EINVAL
    for at in (0, 1, 2, 3):
        assert c.i8_backward_filter(d.handle, *[None if i == at else f for i in range(5)], 0.0, f, big, None) == EINVAL, at
    assert c.i8_backward_filter(d.handle, odd, f, f, f, f, 0.0, f, big, None) == EINVAL
    assert c.i8_backward_filter(plain.handle, f, f, f, f, f, 0.0, f, big, None) == EINVAL  # db of a layer without a bias
    for beta in (0.5, -1.0, float("nan")):
        assert c.i8_backward_filter(d.handle, f, f, f, f, f, beta, f, big, None) == EINVAL
    assert c.i8_backward_filter(none.handle, None, None, None, f, f, 1.0, None, 0, None) == OK
    # w_codes, w_scale, dz, dx
    assert c.i8_backward_data(None, f, f, f, f, f, big, None) == EINVAL
    for at in range(4):
        assert c.i8_backward_data(d.handle, *[None if i == at else f for i in range(4)], f, big, None) == EINVAL, at
    assert c.i8_backward_data(d.handle, odd, f, f, f, f, big, None) == EINVAL
    assert c.i8_backward_data(none.handle, f, f, None, None, None, 0, None) == OK
    for e, call in ((split, lambda w, b: c.i8_backward_filter(split.handle, f, f, f, f, f, 0.0, w, b, None)),
                    (across, lambda w, b: c.i8_backward_data(across.handle, f, f, f, f, w, b, None))):
        need = lib.i8_desc_workspace_bytes(e)
        assert need > 0
        assert call(None, big) == EWORKSPACE and call(f, need - 1) == EWORKSPACE and call(odd, need) == EINVAL


@pytest.mark.parametrize("create,params,field", [(lib.sm_desc_create, dict(rows=4, vocab=100), n) for n in ("rows", "vocab")] +
                         [(lib.i8_desc_create, dict(m=2, k=64, num_output=8), n) for n in ("m", "k", "num_output", "bias_term", "relu")])
def test_parameters_beyond_32_bits_are_refused(create, params, field):
    make = lib.SmParams if create is lib.sm_desc_create else lib.I8Params
    plain = getattr(make(**params), field)
    for value, status in ((plain + (1 << 32), ESHAPE), (plain + (1 << 64), ESHAPE), (plain - (1 << 32), EINVAL)):
        with pytest.raises(lib.ConvError) as e:
            create(make(**{**params, field: value}))
        assert e.value.status == status


# ---- every variant is run by some GPU parity case ----

def test_i8_variants_have_parity_cases():
    import test_i8_parity_gpu as t
    key = lambda m, k, o, dtype: {(re.sub(r"\(W=\d+\)", "", re.sub(r"S=([2-9]|\d\d+)\)", "S)", v)), dtype) for v in
                                  lib.i8_desc_kernel_names(lib.i8_desc_create(lib.I8Params(m, k, o, dtype))).split(";")}
    seen = set().union(*(key(*c[:4]) for c in t.CASES))
    for dtype in (F32, F16, BF16):
        for m in (1, 3, 4, 5, 16, 17, 33, 64, 65, 200, 1000, 1500, 4096, 8192):  # what the library selects over a wide range
            for k in (32, 100, 1024, 4096, 12000, 40000):
                for o in (1, 3, 4, 8, 100, 1000, 2000, 4096, 12000):
                    assert key(m, k, o, dtype) <= seen, (m, k, o, key(m, k, o, dtype) - seen)


def test_i8_input_gradients_of_fp32_never_take_the_tile_that_is_not_built():
    """Whatever the sizes: a round of tiles of 256 counts for 2.3 of those of 128, of which there are twice as many at most."""
    sizes = (4, 8, 100, 255, 256, 257, 512, 1000, 2047, 2048, 4096, 8192, 12000, 16384, 40000, 100000, 130000)
    for m in sizes:
        for k in sizes:
            if m * k < 1 << 30:
                for o in (8, 1000):
                    if max(k, m) * o < 1 << 30:
                        assert "bwd_data=i8_gradient[256" not in lib.i8_desc_kernel_names(lib.i8_desc_create(lib.I8Params(m, k, o, F32)))


def test_sm_layouts_have_parity_cases():
    """What the kernels of a type tell apart: rows that a team holds, rows in segments of one chunk, and of several; each with limits and without, as
    every parity case runs."""
    import inspect

    import test_sm_parity_gpu as t

    def layout(rows, vocab, dtype):
        chunk = 1024 if dtype is F32 else 2048
        size = lib.sm_desc_workspace_bytes(lib.sm_desc_create(lib.SmParams(rows, vocab, dtype)))
        assert size % rows == 0
        segments = size // rows // 32  # 16 bytes and four maxima each
        return ("held" if not size else "one chunk" if segments * chunk >= vocab else "several chunks"), dtype
    want = {(kind, dtype) for kind in ("held", "one chunk", "several chunks") for dtype in (F32, F16, BF16)}
    assert {layout(rows, vocab, dtype) for rows in (1, 500) for vocab in (1, 4096, 8193, 160000, 600000, 1 << 24) for dtype in (F32, F16, BF16)} == want
    assert {layout(*c[:3]) for c in t.CASES + t.LONG_CASES} == want
    runs = inspect.getsource(t.test_parity)
    assert "(None, None, None, None)" in runs and "(scale, k, p, q)" in runs and "test_parity(case)" in inspect.getsource(t.test_parity_of_the_longest_rows)


def test_sm_variants_have_parity_cases():
    import test_sm_parity_gpu as t
    key = lambda rows, vocab, dtype: (re.sub(r"S=\d+", "S", lib.sm_desc_kernel_names(lib.sm_desc_create(lib.SmParams(rows, vocab, dtype)))), dtype)
    seen = {key(*c[:3]) for c in t.CASES}
    for dtype in (F32, F16, BF16):
        for rows in (1, 2, 17, 64, 128, 129, 300, 1000, 5000):
            for vocab in (1, 64, 100, 1000, 4096, 5000, 10000, 20000, 32000, 50257, 70000, 128256, 160000):
                assert key(rows, vocab, dtype) in seen, (rows, vocab, key(rows, vocab, dtype))

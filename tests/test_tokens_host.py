"""Host side of the token policy's operators, without a device: exported names, descriptors, refusals."""
import ctypes
import os
import re

import pytest
import torch

import paper_1810_02272_amd as lib
from paper_1810_02272_amd import binding, gn_binding, lp_binding, q4_binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64
fake = ctypes.c_void_p(256)  # never dereferenced: every call below returns before any launch
EINVAL, ESHAPE, EWORKSPACE, OK = binding.CONV_EINVAL, binding.CONV_ESHAPE, binding.CONV_EWORKSPACE, binding.CONV_OK


@pytest.mark.parametrize("prefix,names", [
    ("lp", {"desc_create", "desc_destroy", "desc_workspace_bytes", "desc_kernel_names", "forward", "backward", "forward_backward"}),
    ("gn", {"desc_create", "desc_destroy", "desc_workspace_bytes", "desc_kernel_names", "clip"}),
    ("q4", {"desc_create", "desc_destroy", "desc_workspace_bytes", "desc_packed_bytes", "desc_kernel_names", "pack", "forward"})])
def test_every_declared_symbol_is_exported_and_bound(prefix, names):
    header = open(os.path.join(ROOT, "include", f"mi355{prefix}.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(rf"\b({prefix}_[a-z0-9_]+)\s*\(", header))
    assert declared == {f"{prefix}_{n}" for n in names}
    c = ctypes.CDLL(lib.library_path())
    for name in declared:
        assert hasattr(c, name) and hasattr(lib, name), name


# ---- every variant is run by some GPU parity case ----

def test_lp_variants_have_parity_cases():
    import test_lp_parity_gpu as t
    seen = set()
    for rows, vocab, dtype, top, entropy, scale, _, _ in t.CASES:
        for v in lib.lp_desc_kernel_names(lib.lp_desc_create(lib.LpParams(rows, vocab, dtype, top, entropy, scale))).split(";"):
            seen.add((re.sub(r"S=\d+", "S", v), dtype))
    for dtype in (F32, F16, BF16):
        for form in ("wave4", "wave8", "solo", "block8", "block16", "block26", "long"):
            for which in ("forward", "forward_backward"):
                assert (f"{which}=lp_row[{form}]", dtype) in seen
        assert ("forward=lp_parts(S)+join", dtype) in seen and ("forward_backward=lp_parts(S)+grad", dtype) in seen
        assert ("backward=lp_grad", dtype) in seen
    for form in ("wave4", "wave8", "block8", "block16", "block26", "long"):  # one type: the others' differ in the conversions alone
        assert (f"forward=lp_row[{form},stream]", BF16) in seen and (f"forward_backward=lp_row[{form},stream]", BF16) in seen
    assert ("backward=lp_grad[stream]", BF16) in seen


def test_q4_variants_have_parity_cases():
    import test_q4_parity_gpu as t
    seen = set()
    for m, k, o, dtype, group, bias, relu in t.CASES:
        name = lib.q4_desc_kernel_names(lib.q4_desc_create(lib.Q4Params(m, k, o, dtype, group, bias, relu)))
        terms, shape, splits = re.fullmatch(r"fwd=(terms\+)?q4\[(.*)\]\(S=(\d+),W=\d+\)", name).groups()
        if dtype is F32 and not terms:
            seen.add(("direct", shape))
        seen.add((shape, int(splits) > 1, dtype is F32))
    for wide in (False, True):
        for shape in ("m16,n16,r1", "m16,n64,r1" if wide else "m16,n32,r1", "m16,n16", "m16,n32", "m16,n64", "m32,n64", "m48,n64", "m64,n64"):
            assert (shape, False, wide) in seen, (shape, wide)
        assert any(len(s) == 3 and s[1] and s[2] is wide for s in seen)
    assert ("direct", "m16,n16,r1") in seen and ("direct", "m16,n16") in seen
    seen = {s for s in seen if len(s) == 3}
    for shape in ("m16,n32,r1,stream", "m16,n64,stream"):
        assert (shape, False, False) in seen
    assert ("m16,n64,r1,stream", False, True) in seen


# ---- log probabilities ----

@pytest.mark.parametrize("bad,status", [(dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(top=-1), EINVAL), (dict(top=65), EINVAL),
                                        (dict(vocab=3, top=4), EINVAL), (dict(entropy=2), EINVAL), (dict(scale=0.0), EINVAL),
                                        (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
                                        (dict(vocab=1 << 30), ESHAPE)])
def test_lp_parameters(bad, status):
    with pytest.raises(lib.ConvError) as e:
        lib.lp_desc_create(lib.LpParams(**{**dict(rows=4, vocab=100, dtype=F32, top=2, entropy=1, scale=1.0), **bad}))
    assert e.value.status == status
    with pytest.raises(TypeError):
        lib.lp_desc_create(lib.LpParams(4, 100, F64))
    with pytest.raises(TypeError):
        lib.lp_desc_create(lib.LpParams(4, 100, torch.int32))


def test_lp_calls():
    c = lp_binding._load()
    d = lib.lp_desc_create(lib.LpParams(4, 100, F32, 2, 1))
    plain = lib.lp_desc_create(lib.LpParams(4, 100, F32, 0, 0))
    parts = lib.lp_desc_create(lib.LpParams(1, 100000, BF16, 2, 1))
    none = lib.lp_desc_create(lib.LpParams(0, 100, F32, 2, 1))
    assert lib.lp_desc_workspace_bytes(parts) > 0 and "parts" in lib.lp_desc_kernel_names(parts)
    assert lib.lp_desc_workspace_bytes(d) == 0
    f = fake
    assert c.lp_desc_create(None, None) == EINVAL and c.lp_desc_destroy(None) == EINVAL and c.lp_desc_workspace_bytes(None, None) == EINVAL
    assert c.lp_desc_kernel_names(None) == b""
    assert c.lp_forward(None, f, 100, f, f, f, f, f, f, f, 0, None) == EINVAL
    assert c.lp_forward(d.handle, None, 100, f, f, f, f, f, f, f, 0, None) == EINVAL      # no logits
    assert c.lp_forward(d.handle, f, 99, f, f, f, f, f, f, f, 0, None) == EINVAL         # rows overlap
    assert c.lp_forward(d.handle, f, 100, None, f, f, f, f, f, f, 0, None) == EINVAL     # logp of what
    assert c.lp_forward(d.handle, f, 100, f, None, f, f, f, f, f, 0, None) == EINVAL
    assert c.lp_forward(d.handle, f, 100, f, f, f, f, None, f, f, 0, None) == EINVAL     # alternatives: both or neither, as described
    assert c.lp_forward(d.handle, f, 100, f, f, f, f, f, None, f, 0, None) == EINVAL
    assert c.lp_forward(d.handle, f, 100, f, f, f, f, None, None, f, 0, None) == EINVAL
    assert c.lp_forward(plain.handle, f, 100, f, f, None, f, f, f, f, 0, None) == EINVAL
    assert c.lp_forward(plain.handle, f, 100, f, f, f, f, None, None, f, 0, None) == EINVAL  # entropy of a descriptor without
    assert c.lp_forward(parts.handle, f, 100000, f, f, f, f, f, f, None, 0, None) == EWORKSPACE
    assert c.lp_forward(parts.handle, f, 100000, f, f, f, f, f, f, f, 8, None) == EWORKSPACE
    assert c.lp_forward(none.handle, None, 0, None, None, None, None, None, None, None, 0, None) == OK
    assert c.lp_backward(None, f, 100, f, f, f, f, f, 100, None) == EINVAL
    for hole in range(7):
        args = [f, 100, f, f, f, f, f, 100]
        at = [0, 1, 2, 3, 4, 6, 7][hole]
        args[at] = 99 if at in (1, 7) else None
        assert c.lp_backward(d.handle, *args, None) == EINVAL, at
    assert c.lp_backward(plain.handle, f, 100, f, f, f, f, f, 100, None) == EINVAL       # d_entropy of a descriptor without
    assert c.lp_backward(none.handle, None, 0, None, None, None, None, None, 0, None) == OK
    assert c.lp_forward_backward(None, f, 100, f, f, f, f, f, f, 100, f, 0, None) == EINVAL
    for at in (0, 1, 2, 3, 7, 8):
        args = [f, 100, f, f, f, f, f, f, 100]
        args[at] = 99 if at in (1, 8) else None
        if at == 7:
            args[7] = None
        assert c.lp_forward_backward(d.handle, *args, f, 0, None) == EINVAL, at
    assert c.lp_forward_backward(plain.handle, f, 100, f, f, f, f, None, f, 100, f, 0, None) == EINVAL
    assert c.lp_forward_backward(plain.handle, f, 100, f, f, None, f, f, f, 100, f, 0, None) == EINVAL
    assert c.lp_forward_backward(parts.handle, f, 100000, f, f, f, f, f, f, 100000, None, 0, None) == EWORKSPACE


@pytest.mark.parametrize("rows", [1 << 22, (1 << 30) - 1, 1 << 30, (1 << 30) + 64, (1 << 31) - 1])
@pytest.mark.parametrize("vocab", [1, 40000, 200000, (1 << 30) - 1])
def test_lp_descriptors_of_any_number_of_rows(rows, vocab):
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, BF16, min(vocab, 64), 1))
    assert "parts" not in lib.lp_desc_kernel_names(d) and lib.lp_desc_workspace_bytes(d) == 0


def test_lp_refuses_cpu_tensors():
    d = lib.lp_desc_create(lib.LpParams(2, 10, F32, 0, 0))
    x, t = torch.zeros(2, 10), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        lib.lp_forward(d, x, t, torch.zeros(2))
    with pytest.raises(TypeError):
        lib.lp_forward_backward(d, x, t, torch.zeros(2), None, None, None, torch.zeros(2, 10))


# ---- clipping ----

def test_gn_parameters_and_calls():
    c = gn_binding._load()
    for counts, dtypes in (([-1], [F32]), ([1 << 40], [F32]), ([1 << 39, 1 << 39], [F32, F32])):
        with pytest.raises(lib.ConvError):
            lib.gn_desc_create(lib.GnParams(counts, dtypes))
    with pytest.raises(lib.ConvError) as e:
        lib.gn_desc_create(lib.GnParams([1] * ((1 << 18) + 1), [F32] * ((1 << 18) + 1)))
    assert e.value.status == ESHAPE
    with pytest.raises(TypeError):
        lib.gn_desc_create(lib.GnParams([1], [torch.int32]))
    with pytest.raises(ValueError):
        lib.GnParams([1, 2], [F32])
    for params in (None, gn_binding._CParams(-1, None, None), gn_binding._CParams(2, None, None)):
        out = ctypes.c_void_p()
        assert c.gn_desc_create(ctypes.byref(out), ctypes.byref(params) if params else None) == EINVAL
    bad = gn_binding._CParams(1, (ctypes.c_int64 * 1)(3), (ctypes.c_int32 * 1)(4))
    assert c.gn_desc_create(ctypes.byref(ctypes.c_void_p()), ctypes.byref(bad)) == EINVAL
    d = lib.gn_desc_create(lib.GnParams([3, 0], [F32, F64]))
    bytes_ = lib.gn_desc_workspace_bytes(d)
    two = (ctypes.c_void_p * 2)(256, None)
    hole = (ctypes.c_void_p * 2)(None, 256)
    assert c.gn_desc_destroy(None) == EINVAL and c.gn_desc_workspace_bytes(None, None) == EINVAL and c.gn_desc_kernel_names(None) == b""
    assert c.gn_clip(None, two, 1.0, two, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, None, 1.0, two, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, two, 1.0, None, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, hole, 1.0, two, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, two, 1.0, hole, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, two, -1.0, two, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, two, float("nan"), two, None, fake, bytes_, None) == EINVAL
    assert c.gn_clip(d.handle, two, 1.0, two, None, None, 0, None) == EWORKSPACE
    assert c.gn_clip(d.handle, two, 1.0, two, None, fake, bytes_ - 1, None) == EWORKSPACE
    with pytest.raises(TypeError):
        lib.gn_clip(d, [torch.zeros(3), torch.zeros(0, dtype=F64)], 1.0)


# ---- 4-bit weights ----

@pytest.mark.parametrize("bad,status", [(dict(m=-1), EINVAL), (dict(k=0), EINVAL), (dict(num_output=0), EINVAL), (dict(group=16), EINVAL),
                                        (dict(group=0), EINVAL), (dict(bias_term=2), EINVAL), (dict(relu=-1), EINVAL),
                                        (dict(k=1 << 15, num_output=1 << 15), ESHAPE), (dict(m=1 << 20, k=1 << 10), ESHAPE),
                                        (dict(m=1 << 20, num_output=1 << 10), ESHAPE)])
def test_q4_parameters(bad, status):
    with pytest.raises(lib.ConvError) as e:
        lib.q4_desc_create(lib.Q4Params(**{**dict(m=2, k=64, num_output=8, dtype=BF16, group=32, bias_term=0, relu=0), **bad}))
    assert e.value.status == status
    with pytest.raises(TypeError):
        lib.q4_desc_create(lib.Q4Params(2, 64, 8, F64))


def test_q4_calls():
    c = q4_binding._load()
    d = lib.q4_desc_create(lib.Q4Params(2, 64, 8, BF16, 32, 1, 0))
    plain = lib.q4_desc_create(lib.Q4Params(2, 64, 8, BF16, 32, 0, 0))
    none = lib.q4_desc_create(lib.Q4Params(0, 64, 8, BF16, 32, 0, 0))
    assert lib.q4_desc_packed_bytes(d) >= 8 * 64 // 2 and lib.q4_desc_packed_bytes(d) == lib.q4_desc_packed_bytes(none)
    f, odd = fake, ctypes.c_void_p(264)
    assert c.q4_desc_create(None, None) == EINVAL and c.q4_desc_destroy(None) == EINVAL
    assert c.q4_desc_packed_bytes(None, None) == EINVAL and c.q4_desc_workspace_bytes(None, None) == EINVAL
    assert c.q4_desc_kernel_names(None) == b""
    assert c.q4_pack(None, f, f, f, None) == EINVAL
    for args in ((None, f, f), (f, None, f), (f, f, None), (f, f, odd)):
        assert c.q4_pack(d.handle, *args, None) == EINVAL
    assert c.q4_forward(None, f, f, f, f, f, 1 << 30, None) == EINVAL
    for args in ((None, f, f, f), (f, None, f, f), (f, f, None, f), (f, f, f, None), (f, odd, f, f)):
        assert c.q4_forward(d.handle, *args, f, 1 << 30, None) == EINVAL
    assert c.q4_forward(plain.handle, f, f, f, f, f, 1 << 30, None) == EINVAL  # bias unexpected
    assert c.q4_forward(none.handle, None, f, None, None, None, 0, None) == OK


@pytest.mark.parametrize("create,params,field", [(lib.lp_desc_create, dict(rows=4, vocab=100, top=2), f) for f in ("rows", "vocab", "top", "entropy")] +
                         [(lib.q4_desc_create, dict(m=2, k=64, num_output=8), f) for f in ("m", "k", "num_output", "group", "bias_term", "relu")])
def test_parameters_beyond_32_bits_are_refused(create, params, field):
    make = lib.LpParams if create is lib.lp_desc_create else lib.Q4Params
    plain = getattr(make(**params), field)
    for value, status in ((plain + (1 << 32), ESHAPE), (plain + (1 << 64), ESHAPE), (plain - (1 << 32), EINVAL)):
        with pytest.raises(lib.ConvError) as e:
            create(make(**{**params, field: value}))
        assert e.value.status == status


def test_gn_counts_beyond_64_bits_are_refused():
    for count, status in (((1 << 64) + 1, ESHAPE), (1 - (1 << 64), EINVAL)):
        with pytest.raises(lib.ConvError) as e:
            lib.gn_desc_create(lib.GnParams([3, count], [F32, F32]))
        assert e.value.status == status


def test_gn_reads_an_iterator_of_gradients_once():
    d = lib.gn_desc_create(lib.GnParams([0, 0], [F32, BF16]))  # of no elements: they may be absent
    for grads in ([None, None], (None, None), iter([None, None]), (t for t in (None, None))):
        with pytest.raises(lib.ConvError) as e:
            lib.gn_clip(d, grads, 1.0, stream=0)
        assert e.value.status == EWORKSPACE  # every tensor found, in place
    with pytest.raises(ValueError):
        lib.gn_clip(d, iter([None]), 1.0, stream=0)


def test_gn_variants_have_parity_cases():
    """The kernels go by the runs of tensors that follow each other (8 and 96 to a launch), by fp64 tensors, and by the bytes of the gradients, and
    of them and outputs elsewhere, against the 256 MB of the last-level cache."""
    import test_gn_parity_gpu as t
    size = {F32: 4, F16: 2, BF16: 2, F64: 8}
    sums, scales, launches = set(), set(), 0
    for (counts, dtypes), apart in [(c, a) for c in (t.ONE, t.MIXED, t.MANY, t.LARGE) for a in (0, 3)] + [(t.HUGE, 0), (t.EVERY_TYPE, 1)] + t.LARGE_CASES:
        used = [(n, d) for n, d in zip(counts, dtypes) if n]
        runs = len(used) if apart else len({d for _, d in used})
        read = sum(n * size[d] for n, d in used)
        table = [8 if min(96, runs - first) <= 8 else 96 for first in range(0, runs, 96)]
        sums |= {(k, read > 1 << 28, F64 in dtypes) for k in table}
        for written in (read, 0):  # outputs elsewhere, in place
            scales |= {(k, read > 1 << 28, read + written > 1 << 28) for k in table}
        if read > 1 << 28:
            launches = max(launches, len(table))
    assert sums == {(k, stream, wide) for k in (8, 96) for stream in (False, True) for wide in (False, True)}
    assert scales == {(k, *s) for k in (8, 96) for s in ((False, False), (False, True), (True, True))}
    assert launches > 2


def test_q4_variants_have_parity_cases_prepared_and_direct():
    """Each shape that fp32 rows may take as they are and as operands laid out before, of each group size; batches beyond 64 rows of each type."""
    import test_q4_parity_gpu as t
    name = lambda m, k, o, dtype, group: lib.q4_desc_kernel_names(lib.q4_desc_create(lib.Q4Params(m, k, o, dtype, group)))
    key = lambda text: re.sub(r"\(S=\d+,W=\d+\)", "", text)
    cases = t.CASES + t.MORE_CASES
    seen = {(key(name(*c[:5])), c[3]) for c in cases}
    for m in (1, 4, 5, 16, 17, 33, 49, 64):  # what the library selects over a wide range
        for k in (32, 100, 1024, 1025, 4096, 12000):
            for o in (8, 100, 4096, 4097, 8000, 16384, 20000, 33000):
                for dtype in (F32, F16, BF16):
                    n = key(name(m, k, o, dtype, 64))
                    assert (n, dtype) in seen or dtype is not F32 and (n, BF16 if dtype is F16 else F16) in seen, (n, dtype, m, k, o)
    prepared = {(key(name(*c[:5])), c[4]) for c in t.MORE_CASES if c[3] is F32 and c[0] <= 16}
    assert prepared >= {(f"fwd=terms+q4[{shape}]", group) for shape in ("m16,n16,r1", "m16,n32") for group in (32, 64, 128)}
    assert {c[3] for c in cases if c[0] > 64} == {F32, F16, BF16}


def test_lp_row_kernels_of_parts_are_those_that_are_launched():
    """Parts of a row are taken by workgroups of 1024 threads, through the cache; the library holds no kernel of them for another team."""
    with open(lib.library_path(), "rb") as f:
        built = re.findall(rb"lp_row_kernelILi(\d)ELi(\d+)ELi(\d+)ELN\w*?4ModeE(\d)ELb([01])ELb([01])E", f.read())
    kernels = {tuple(map(int, k)) for k in built}  # type, threads, vectors, mode (2: a part), entropy, stream
    assert {k for k in kernels if k[3] == 2} == {(t, 1024, 4, 2, e, 0) for t in (0, 1, 2) for e in (0, 1)}
    teams = {(64, 4), (64, 8), (256, 8), (256, 16), (256, 26), (512, 20)}
    assert {k[1:3] + k[5:] for k in kernels if k[3] < 2} == {(*team, stream) for team in teams for stream in (0, 1)} | {(1024, 4, 0)}


@pytest.mark.parametrize("group", [32, 64, 128])
def test_q4_codes_go_around_the_cache_by_the_packed_size(group):
    """As the logits and gradients of the other operators do: where there is more than the 256 MB that the last-level cache holds."""
    seen = set()
    for o in range(100000, 136000, 512):
        d = lib.q4_desc_create(lib.Q4Params(1, 4096, o, BF16, group))
        large = lib.q4_desc_packed_bytes(d) > 1 << 28
        assert ("stream" in lib.q4_desc_kernel_names(d)) == large, o
        seen.add(large)
    assert seen == {False, True}


def test_lp_long_rows_take_the_denser_team_from_a_thousand_rows_on():
    """Three teams on a compute unit: measured faster, or as fast within 7 %, for any number of rows beyond 1024 (at 2400 they were not taken)."""
    team = lambda rows: re.search(r"forward=lp_row\[(\w+)", lib.lp_desc_kernel_names(lib.lp_desc_create(lib.LpParams(rows, 50257, BF16, 20, 1)))).group(1)
    assert {team(rows) for rows in range(1025, 9000, 7)} == {"block26"}
    assert team(512) == "long" and team(768) == "block26" and team(777) == "long"

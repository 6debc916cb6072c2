"""The gradient norm and clipping (include/mi355gn.h) against the oracle in 64 bits.

Tolerances: squares and sums are held in fp64, so the norm is off by its rounding to fp32 (2^-24); the factor by its rounding to fp32 (2^-24;
none for fp64 tensors), the product by its own in fp32 (2^-24) and by the output type's half step."""
import math

import pytest
import torch

import paper_1810_02272_amd as lib
from oracle import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64


def views(counts, dtypes, apart, first, fill):
    """Tensors one after the other in a buffer for each type, `apart` elements between them, and the buffers."""
    size = {t: first + sum(n + apart for n, u in zip(counts, dtypes) if u is t) + 8 for t in set(dtypes)}
    buffers = {t: torch.full((n,), math.nan, device=DEV, dtype=t) for t, n in size.items()}
    at = {t: first for t in size}
    out = []
    for n, t in zip(counts, dtypes):
        v = buffers[t][at[t]:at[t] + n]
        v.copy_(fill(n).to(t))
        out.append(v)
        at[t] += n + apart
    return out, buffers


def rest_untouched(tensors, buffers):
    for t, b in buffers.items():
        rest = torch.ones_like(b, dtype=torch.bool)
        for v in tensors:
            if v.dtype is t:
                rest[v.storage_offset():v.storage_offset() + v.numel()] = False
        assert torch.isnan(b[rest]).all()


def check(norm, outs, grads, limit):
    want_norm, want = tokens.clip(grads, limit)
    assert abs(float(norm) - want_norm) <= 2.0 ** -23 * want_norm
    for o, w, g in zip(outs, want, grads):
        if want_norm <= limit:
            assert torch.equal(o, g)
            continue
        eps = torch.finfo(o.dtype).eps
        small = {F16: 2.0 ** -25, F64: 0.0}.get(o.dtype, 2.0 ** -126)
        steps = 2.0 ** -51 if o.dtype is F64 else 2.0 ** -23
        assert bool(((o.double() - w).abs() <= w.abs() * (eps / 2 + steps) + small).all()), (o.dtype, o.numel())


ONE = ([1], [F32])
MIXED = ([5, 0, 1, 4097, 3, 65537, 16, 8, 70000], [F32, BF16, BF16, F16, F64, BF16, F32, F32, F64])
MANY = ([(i * 37) % 301 for i in range(400)], [(F32, F16, BF16, F64)[i * i % 4] for i in range(400)])
HUGE = ([70000001, 3, 40000000], [BF16, F32, F32])  # more than the last-level cache holds
LARGE = ([3000001, 17, 5000000, 2000003], [BF16, BF16, F32, BF16])


@pytest.mark.parametrize("counts,dtypes", [ONE, MIXED, MANY, LARGE], ids=["one", "mixed", "many", "large"])
@pytest.mark.parametrize("apart,first", [(0, 0), (0, 1), (3, 0), (1, 1)])
@pytest.mark.parametrize("ratio", [0.3, 0.0, 7.0])
def test_parity(counts, dtypes, apart, first, ratio):
    g = torch.Generator(device=DEV).manual_seed(len(counts))
    fill = lambda n: torch.randn(n, generator=g, device=DEV)
    grads, grad_buffers = views(counts, dtypes, apart, first, fill)
    outs, out_buffers = views(counts, dtypes, apart, first, lambda n: torch.full((n,), math.nan, device=DEV))
    limit = ratio * math.sqrt(sum(counts))
    d = lib.gn_desc_create(lib.GnParams(counts, dtypes))
    bytes_ = lib.gn_desc_workspace_bytes(d)
    ws = torch.full((bytes_ // 4 + 16,), math.nan, device=DEV)
    norm = torch.full((1,), math.nan, device=DEV)
    lib.gn_clip(d, grads, limit, outs, norm, ws[:bytes_ // 4])
    assert torch.isnan(ws[bytes_ // 4:]).all()
    check(norm, outs, grads, limit)
    rest_untouched(outs, out_buffers)
    again = [torch.empty_like(t) for t in outs]
    lib.gn_clip(d, grads, limit, again, None, ws)        # separate tensors: the sums' order may differ, not the values by more than it
    check(norm, again, grads, limit)
    before = [t.clone() for t in grads]
    lib.gn_clip(d, tuple(grads), limit, None, norm, ws)  # in place
    check(norm, grads, before, limit)
    rest_untouched(grads, grad_buffers)
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.parametrize("first", [0, 1])
@pytest.mark.parametrize("ratio", [0.3, 7.0])
def test_more_than_the_cache_holds(first, ratio):
    test_parity(*HUGE, 0, first, ratio)


def run(grads, limit):
    d = lib.gn_desc_create(lib.GnParams([t.numel() for t in grads], [t.dtype for t in grads]))
    ws = torch.empty(lib.gn_desc_workspace_bytes(d) // 4, device=DEV)
    norm, outs = torch.empty(1, device=DEV), [torch.empty_like(t) for t in grads]
    lib.gn_clip(d, grads, limit, outs, norm, ws)
    return float(norm), outs


def test_extremes():
    big = torch.full((1000,), 1e30, device=DEV)
    norm, (out,) = run([big], 1.0)
    assert norm == pytest.approx(1e30 * math.sqrt(1000), rel=1e-6) and torch.allclose(out, torch.full_like(out, 1000 ** -0.5))
    tiny = torch.full((1000,), 1e-30, device=DEV)
    norm, (out,) = run([tiny], 1.0)
    assert norm == pytest.approx(1e-30 * math.sqrt(1000), rel=1e-6) and torch.equal(out, tiny)
    zero = torch.zeros(77, device=DEV, dtype=BF16)
    norm, (out,) = run([zero], 0.0)
    assert norm == 0.0 and torch.equal(out, zero)
    nan = torch.ones(50, device=DEV)
    nan[7] = math.nan
    norm, (out,) = run([nan], 1.0)
    assert math.isnan(norm) and torch.equal(out.nan_to_num(9.0), nan.nan_to_num(9.0))
    inf = torch.ones(50, device=DEV)
    inf[7] = -math.inf
    norm, (out,) = run([inf], 1.0)
    assert norm == math.inf and math.isnan(float(out[7])) and float(out[0]) == 0.0
    norm, (out,) = run([big], math.inf)
    assert torch.equal(out, big)
    assert run([], 1.0)[0] == 0.0
    assert run([torch.empty(0, device=DEV), torch.empty((0, 3), device=DEV, dtype=F16)], 1.0)[0] == 0.0


def test_shapes_are_free_and_a_norm_is_that_of_all():
    grads = [torch.randn(3, 4, 5, device=DEV), torch.randn(7, device=DEV, dtype=F64), torch.randn(64, 64, device=DEV).to(BF16)]
    norm, outs = run(grads, 2.0)
    check(norm, outs, grads, 2.0)
    assert abs(math.sqrt(sum(float(t.double().square().sum()) for t in outs)) - 2.0) < 2.0 * 2.0 ** -8


def test_in_a_graph():
    grads = [torch.randn(1000, device=DEV), torch.randn(333, device=DEV)]
    d = lib.gn_desc_create(lib.GnParams([1000, 333], [F32, F32]))
    ws = torch.empty(lib.gn_desc_workspace_bytes(d) // 4, device=DEV)
    norm, outs = torch.empty(1, device=DEV), [torch.empty_like(t) for t in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lib.gn_clip(d, grads, 3.0, outs, norm, ws, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.gn_clip(d, grads, 3.0, outs, norm, ws)
    for k in range(3):
        for t in grads:
            t.normal_()
        graph.replay()
        replayed = [norm.clone()] + [t.clone() for t in outs]
        check(norm, outs, grads, 3.0)
        lib.gn_clip(d, grads, 3.0, outs, norm, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, [norm] + outs))


def test_refusals_on_the_device():
    d = lib.gn_desc_create(lib.GnParams([4, 6], [F32, BF16]))
    a, b = torch.zeros(4, device=DEV), torch.zeros((2, 3), device=DEV, dtype=BF16)
    ws = torch.empty(lib.gn_desc_workspace_bytes(d) // 4, device=DEV)
    lib.gn_clip(d, [a, b], 1.0, ws=ws)
    lib.gn_clip(d, iter([a, b]) and [a, b], 1, (a, b), None, ws)
    for grads, limit, outs, space, error in (([a], 1.0, None, ws, ValueError), ([a, b.float()], 1.0, None, ws, TypeError),
                                             ([a, b[:1]], 1.0, None, ws, ValueError), ([a, b.t()], 1.0, None, ws, TypeError),
                                             ([a, b.cpu()], 1.0, None, ws, TypeError), ([a, b], -1.0, None, ws, lib.ConvError),
                                             ([a, b], math.nan, None, ws, lib.ConvError), ([a, None], 1.0, None, ws, lib.ConvError),
                                             ([a, b], 1.0, [a, None], ws, lib.ConvError), ([a, b], 1.0, None, None, lib.ConvError),
                                             ([a, b], 1.0, None, ws[:-1], lib.ConvError)):
        with pytest.raises(error):
            lib.gn_clip(d, grads, limit, outs, None, space)


def test_gradients_from_an_iterator():
    grads = [torch.randn(300, device=DEV), torch.randn((2, 3), device=DEV).to(BF16)]
    d = lib.gn_desc_create(lib.GnParams([300, 6], [F32, BF16]))
    ws, norm = torch.empty(lib.gn_desc_workspace_bytes(d) // 4, device=DEV), torch.empty(1, device=DEV)
    before = [t.clone() for t in grads]
    lib.gn_clip(d, iter(grads), 3.0, None, norm, ws)
    check(norm, grads, before, 3.0)
    outs = [torch.empty_like(t) for t in grads]
    lib.gn_clip(d, (t for t in before), 3.0, (t for t in outs), norm, ws)
    check(norm, outs, before, 3.0)


def scaled_clip(grads, limit):
    """(norm, outputs) in 64 bits, the squares taken of values over the greatest: none overflows or vanishes."""
    most = max(float(g.double().abs().max()) for g in grads)
    norm = most * math.sqrt(math.fsum(float((g.double() / most).square().sum()) for g in grads))
    factor = lambda g: g.double() / norm * limit if norm > limit else g.double()  # (limit / norm itself may be out of range)
    return norm, [factor(g) for g in grads]


def check_scaled(grads, limit):
    norm, outs = run(grads, limit)
    want_norm, want = scaled_clip(grads, limit)
    assert norm == pytest.approx(float(torch.tensor(want_norm, dtype=F64).float()), rel=2.0 ** -23, abs=2.0 ** -149)
    for o, w, g in zip(outs, want, grads):
        if want_norm <= limit:
            assert torch.equal(o, g)
            continue
        info = torch.finfo(o.dtype)
        steps = 2.0 ** -50 if o.dtype is F64 else 2.0 ** -23  # fp64: the norm's sum and root, the factor, the product; here in the oracle too
        bound = w.abs() * (info.eps / 2 + steps) + (2.0 ** -25 if o.dtype is F16 else 2.0 ** -126 if o.dtype is not F64 else 0.0)
        assert bool(((o.double() - w).abs() <= bound).all()), (o.dtype, o.numel())


@pytest.mark.parametrize("size,limit", [(3e38, 1.0), (1e30, 1e-15), (1e25, 1e-20), (1e38, 1e-3), (1e20, 1e-18)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_factors_below_the_normal_range(dtype, size, limit):
    """The limit over the norm is subnormal in fp32, or less; the products are not."""
    g = torch.Generator(device=DEV).manual_seed(1)
    sign = lambda n: torch.randint(2, (n,), generator=g, device=DEV) * 2.0 - 1.0
    check_scaled([(sign(1000) * size).to(dtype), (torch.rand(4099, generator=g, device=DEV) * size).to(dtype)], limit)
    check_scaled([(torch.rand(70001, generator=g, device=DEV) * size).to(dtype), torch.randn(77, generator=g, device=DEV).to(F16),
                  torch.randn(500, generator=g, device=DEV, dtype=F64) * size], limit)


@pytest.mark.parametrize("exponent", [300, 200, 160, -100, -160, -200, -290])
@pytest.mark.parametrize("ratio", [0.3, 3.0])
def test_fp64_gradients_whose_squares_leave_the_range(exponent, ratio):
    g = torch.Generator(device=DEV).manual_seed(2)
    r = lambda n: torch.randn(n, generator=g, device=DEV, dtype=F64) * 10.0 ** exponent
    for n in (1, 3, 1001, 2000003):
        check_scaled([r(n)], ratio * math.sqrt(n) * 10.0 ** exponent)
    check_scaled([r(5000), torch.randn(333, generator=g, device=DEV), r(77)], ratio * math.sqrt(5077) * 10.0 ** exponent)


@pytest.mark.parametrize("at", [478, 479, 480, 481, 482, -478, -479, -480, -481, -482])
def test_fp64_gradients_of_two_ranges_count_alike(at):
    """Magnitudes on both sides of a power of two, each a good part of the norm."""
    g = torch.Generator(device=DEV).manual_seed(3)
    t = torch.ldexp(torch.rand(3001, generator=g, device=DEV, dtype=F64) * 3 + 0.25, torch.tensor(at, device=DEV)).contiguous()
    check_scaled([t[:1000], t[1000:], torch.zeros(5, device=DEV)], 2.0 ** at)
    check_scaled([t, torch.ones(3, device=DEV)], 2.0 ** at)


def test_fp64_infinities_and_zeros():
    zero = torch.zeros(77, device=DEV, dtype=F64)
    norm, (out,) = run([zero], 0.0)
    assert norm == 0.0 and torch.equal(out, zero)
    big = torch.full((50,), 1e300, device=DEV, dtype=F64)
    for bad in (math.inf, -math.inf):
        big[7] = bad
        norm, (out,) = run([big], 1.0)
        assert norm == math.inf and math.isnan(float(out[7])) and float(out[0]) == 0.0
    for size in (1e300, 1.0, 1e-300):
        nan = torch.full((50,), size, device=DEV, dtype=F64)
        nan[7] = math.nan
        norm, (out,) = run([nan], 1.0)
        assert math.isnan(norm) and torch.equal(out.nan_to_num(9.0), nan.nan_to_num(9.0))


# Every kernel beyond the small sizes above: tables of up to 8 and up to 96 runs, with fp64 tensors and without, the sum around the cache, the
# product with reads, or writes alone, around it; what the second pass finds in the cache over several launches.
FEW_OUT = ([20000003, 30000001, 17], [F32, BF16, F32])
FEW_HUGE = ([30000001, 5, 20000003], [F64, F32, BF16])
MANY_OUT = ([1200003 + 1000 * i for i in range(40)], [(F32, BF16)[i % 3 == 2] for i in range(40)])
MANY_HUGE = ([8000009 + 16 * i for i in range(12)], [(F32, F32, F64, BF16)[i % 4] for i in range(12)])
LAUNCHES = ([600011 + (i * 37) % 301 for i in range(250)], [(F32, BF16)[i % 5 == 4] for i in range(250)])
EVERY_TYPE = ([(i * 53) % 1009 for i in range(130)], [(F32, F16, BF16, F64)[i % 4] for i in range(130)])
LARGE_CASES = [(FEW_OUT, 0), (FEW_HUGE, 0), (MANY_OUT, 3), (MANY_HUGE, 5), (LAUNCHES, 1)]


@pytest.mark.parametrize("case,apart", LARGE_CASES, ids=["few-out", "few-huge", "many-out", "many-huge", "launches"])
@pytest.mark.parametrize("ratio", [0.3, 7.0])
def test_large_calls(case, apart, ratio):
    test_parity(*case, apart, 1, ratio)


@pytest.mark.parametrize("ratio", [0.3, 7.0])
def test_every_type_over_several_launches(ratio):
    """fp64 outputs, with u = 2^-53: a square is rounded and passes at most 32 additions of such (a thread's chunk 6, a wave 6, four waves 4, the parts
    1, 6, 4 and 4 more where a launch has more chunks than one), 33 u in all, half of that in the root, and the root, the factor and the
    product are rounded: 20 u.  The oracle's sum is exact."""
    counts, dtypes = EVERY_TYPE
    g = torch.Generator(device=DEV).manual_seed(len(counts))
    grads, _ = views(counts, dtypes, 1, 1, lambda n: torch.randn(n, generator=g, device=DEV))
    outs, out_buffers = views(counts, dtypes, 1, 1, lambda n: torch.full((n,), math.nan, device=DEV))
    limit = ratio * math.sqrt(sum(counts))
    d = lib.gn_desc_create(lib.GnParams(counts, dtypes))
    ws, norm = torch.empty(lib.gn_desc_workspace_bytes(d) // 4, device=DEV), torch.empty(1, device=DEV)
    lib.gn_clip(d, grads, limit, outs, norm, ws)
    want = math.sqrt(math.fsum(v * v for t in grads for v in t.double().tolist()))
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    rest_untouched(outs, out_buffers)
    for o, t in zip(outs, grads):
        if want <= limit:
            assert torch.equal(o, t)
            continue
        w = t.double() * (limit / want)
        steps = 20 * 2.0 ** -53 if o.dtype is F64 else 2.0 ** -23 + torch.finfo(o.dtype).eps / 2
        small = {F16: 2.0 ** -25, F64: 0.0}.get(o.dtype, 2.0 ** -126)
        assert bool(((o.double() - w).abs() <= w.abs() * steps + small).all()), (o.dtype, o.numel())
    lib.gn_clip(d, grads, limit, None, norm, ws)  # in place
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.parametrize("size", [1e-300, 1e-200, 1e-30, 1.0, 1e200])
def test_fp64_value_among_zeros(size):
    """One value, wherever it stands, among zeros of both signs: the norm is its size."""
    n = 2 * 2048 + 3  # two chunks and an odd end
    for at in (0, 1, 2, 511, 2047, 2048, 4095, n - 3, n - 2, n - 1):
        t = torch.zeros(n, device=DEV, dtype=F64)
        t[1::2] = -0.0
        t[at] = -size
        check_scaled([t], size / 4)
        check_scaled([t], size * 4)

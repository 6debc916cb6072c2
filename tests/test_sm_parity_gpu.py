"""Drawing tokens (include/mi355sm.h) against the oracle in 64 bits.

Tokens are whole numbers and have to be equal: weights and sums are held in 64 bits on both sides, and none of these inputs has a border within
2^-40 of the whole of u or p, but for those made to meet one exactly, with weights that are powers of two.  Log probabilities: an exponent of 64
bits, a logarithm and one rounding to fp32, half a step (2^-24 relative)."""
import math

import pytest
import torch

import paper_1810_02272_amd as lib
from oracle import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
I32 = torch.int32

# rows, vocab, dtype, stride, spread of the logits
CASES = [
    (1, 1, F32, 1, 1.0), (1, 1, BF16, 1, 1.0), (3, 2, F16, 5, 1.0), (5, 7, BF16, 7, 2.0), (64, 8, F32, 8, 2.0), (33, 9, F16, 11, 2.0), (200, 64, BF16, 64, 3.0),
    (50, 255, F32, 300, 1.0), (40, 1000, F16, 1001, 3.0), (60, 4096, F32, 4096, 2.0), (30, 4097, F32, 4097, 2.0), (30, 8192, BF16, 8192, 3.0), (20, 8193, F16, 8193, 3.0),
    (10, 32000, BF16, 32000, 2.0), (6, 50257, F16, 50304, 4.0), (4, 65537, BF16, 65537, 1.0), (3, 131072, BF16, 131073, 3.0), (2, 128256, F32, 128256, 2.0),
    (2, 160001, F16, 160001, 2.0), (1, 700000, BF16, 700000, 3.0), (300, 3000, BF16, 3000, 0.1), (12, 20000, BF16, 20000, 0.02), (600, 128, BF16, 128, 3.0),
]
SCALES, KS = (0.25, 0.75, 1.0, 1.25, 3.0), (0, 0, 1, 2, 5, 40, 1000, 5000, 1 << 30, -3)
PS, QS = (1.0, 1.0, 0.0, 0.3, 0.9, 0.95, 0.999, 2.0), (0.0, 0.0, 0.01, 0.1, 0.7, 1.0, 3.0, -1.0)


def make(case, seed=0):
    rows, vocab, dtype, stride, spread = case
    g = torch.Generator(device=DEV).manual_seed(seed + rows * vocab)
    x = torch.full((rows, stride), math.nan, device=DEV, dtype=dtype)
    z = torch.randn((rows, vocab), generator=g, device=DEV) * spread
    x[:, :vocab] = (z - 0.6 * torch.log1p(torch.rand((rows, vocab), generator=g, device=DEV) * vocab)).to(dtype)
    pick = lambda values, t=F32: torch.tensor(values, device=DEV, dtype=t)[torch.randint(len(values), (rows,), generator=g, device=DEV)]
    return x[:, :vocab], torch.rand(rows, generator=g, device=DEV), pick(SCALES), pick(KS, I32), pick(PS), pick(QS)


def run(x, u, scale=None, top_k=None, top_p=None, min_p=None, want_logp=True):
    rows, vocab = x.shape
    d = lib.sm_desc_create(lib.SmParams(rows, vocab, x.dtype))
    print(lib.sm_desc_kernel_names(d), flush=True)
    size = lib.sm_desc_workspace_bytes(d)
    ws = torch.full(((size + 3) // 4 + 16,), math.nan, device=DEV)
    token, logp = torch.full((rows + 8,), -77, device=DEV, dtype=I32), torch.full((rows + 8,), 55.0, device=DEV)
    call = lambda t, l: lib.sm_sample(d, x, u, scale, top_k, top_p, min_p, t, l, ws[:(size + 3) // 4])
    call(token[:rows], logp[:rows])
    assert bool((token[rows:] == -77).all()) and bool((logp[rows:] == 55.0).all()) and bool(torch.isnan(ws[(size + 3) // 4:]).all())
    again = torch.empty_like(token[:rows])
    call(again, None)
    assert torch.equal(again, token[:rows])
    return token[:rows], logp[:rows]


def full(rows, value, t=F32):
    return torch.full((rows,), value, device=DEV, dtype=t)


def check(got, x, u, scale=None, top_k=None, top_p=None, min_p=None):
    rows = x.shape[0]
    token, logp = got
    want, want_logp = tokens.draw(x, u, full(rows, 1.0) if scale is None else scale, full(rows, 0, I32) if top_k is None else top_k,
                                  full(rows, 1.0) if top_p is None else top_p, full(rows, 0.0) if min_p is None else min_p)
    assert torch.equal(token, want), [(int(r), int(token[r]), int(want[r])) for r in (token != want).nonzero()[:5, 0]]
    assert bool(((logp.double() - want_logp).abs() <= want_logp.abs() * 1.01 * 2.0 ** -24 + 2.0 ** -45).all())


@pytest.mark.parametrize("case", CASES, ids=["%dx%d-%s-%d-%g" % (c[0], c[1], str(c[2])[6:], c[3], c[4]) for c in CASES])
def test_parity(case):
    x, u, scale, k, p, q = make(case)
    for limits in ((None, None, None, None), (scale, None, None, None), (scale, k, None, None), (scale, None, p, None), (None, None, None, q),
                   (scale, k, p, None), (scale, k, p, q)):
        check(run(x, u, *limits), x, u, *limits)


# segments of several chunks
LONG_CASES = [(2, 300001, F32, 300001, 2.0), (3, 262145, F32, 262147, 0.5), (2, 540001, F16, 540004, 3.0), (2, 1600003, BF16, 1600003, 1.0)]


@pytest.mark.parametrize("case", LONG_CASES, ids=["%dx%d-%s" % (c[0], c[1], str(c[2])[6:]) for c in LONG_CASES])
def test_parity_of_the_longest_rows(case):
    test_parity(case)


@pytest.mark.parametrize("case", CASES + LONG_CASES, ids=["%dx%d-%s" % (c[0], c[1], str(c[2])[6:]) for c in CASES + LONG_CASES])
def test_no_case_has_a_border_within_what_the_arithmetic_may_be_off(case):
    """Of the whole, u and p are 2^-40 or more away from every sum that decides about them, and of q every weight that is not equal to it."""
    x, u, scale, k, p, q = make(case)
    rows, vocab = x.shape
    for limits in ((None, None, None, None), (scale, None, None, None), (scale, k, None, None), (scale, None, p, None), (None, None, None, q),
                   (scale, k, p, None), (scale, k, p, q)):
        s, kk, pp, qq = (t if t is not None else full(rows, v, d) for t, v, d in zip(limits, (1.0, 0, 1.0, 0.0), (F32, I32, F32, F32)))
        by, index = torch.sort(x.double(), dim=1, descending=True, stable=True)
        by = torch.exp((by - by[:, :1]) * s.double()[:, None])
        place = torch.arange(vocab, device=DEV)[None]
        by = torch.where((place < kk[:, None]) | (kk <= 0)[:, None], by, 0.0)
        sums = by.cumsum(1)
        target = pp.double()[:, None] * sums[:, -1:]
        limited = ((pp > 0) & (pp < 1))[:, None] & (place < vocab)
        assert bool(((sums - target).abs() > sums[:, -1:] * 2.0 ** -40)[limited].all())
        by = torch.where((place <= (sums < target).sum(1, keepdim=True)) | (pp >= 1)[:, None], by, 0.0)
        least = qq.double().clamp(max=1.0)[:, None]
        assert bool(((by == least) | ((by - least).abs() > least * 2.0 ** -40))[(qq > 0)[:, None] & (by > 0)].all())
        kept = torch.zeros_like(by).scatter_(1, index, torch.where((by >= least) | (qq <= 0)[:, None], by, 0.0))
        sums = kept.cumsum(1)
        near = ((sums - u.double()[:, None] * sums[:, -1:]).abs() <= sums[:, -1:] * 2.0 ** -40) & (kept > 0)
        assert not bool(near.any())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_against_the_definition_token_by_token(dtype):
    x, u, scale, k, p, q = make((120, 37, dtype, 40, 2.0), seed=4)
    x[5, 3:] = -math.inf
    x[6, :36] = -math.inf
    x[7] = 0.5
    x[8, ::2], x[8, 1::2] = 0.0, -0.0
    token, logp = run(x, u, scale, k, p, q)
    for r in range(120):
        want = tokens.draw_row(x[r].cpu(), float(u[r]), float(scale[r]), int(k[r]), float(p[r]), float(q[r]))
        assert int(token[r]) == want[0], r
        assert abs(float(logp[r]) - want[1]) <= 1e-6 * (1 + abs(want[1]))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [1, 6, 5000, 70000])
def test_rows_without_a_distribution_and_bad_parameters(dtype, vocab):
    rows = 16
    x = torch.randn((rows, vocab), device=DEV).to(dtype)
    u, scale, k, p, q = full(rows, 0.5), full(rows, 1.0), full(rows, 3, I32), full(rows, 0.9), full(rows, 0.1)
    x[0], x[1, vocab - 1], x[2, 0] = -math.inf, math.nan, math.inf
    x[3], x[4] = math.nan, math.inf
    scale[5], scale[6], scale[7], scale[8] = 0.0, math.nan, -1.0, math.inf
    u[9], u[10], u[11] = -0.001, 1.001, math.nan
    p[12], q[13] = math.nan, math.nan
    scale[14] = 2.0 ** 61
    token, logp = run(x, u, scale, k, p, q)
    assert bool((token[:15] == -1).all()) and int(token[15]) >= 0
    assert float(logp[0]) == -math.inf and bool(torch.isnan(logp[1:15]).all()) and math.isfinite(float(logp[15]))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [3, 1000, 33000, 140000])
def test_banned_tokens_are_never_drawn(dtype, vocab):
    rows = 40
    x = torch.randn((rows, vocab), device=DEV).to(dtype)
    allowed = torch.randint(vocab, (rows,), device=DEV)
    x.fill_(-math.inf)
    x[torch.arange(rows, device=DEV), allowed] = 1.0
    u = torch.linspace(0, 1, rows, device=DEV)
    for limits in ((None, None, None, None), (None, full(rows, 2, I32), None, None), (None, None, full(rows, 0.5), None), (None, full(rows, 2, I32), full(rows, 0.99), full(rows, 0.5))):
        token, logp = run(x, u, *limits)
        assert torch.equal(token, allowed.int()) and bool((logp == 0).all())
    low = torch.finfo(dtype).min
    x = torch.where(x == 1.0, x, torch.full_like(x, low))  # finite masks
    token, _ = run(x, u, full(rows, 1.0), full(rows, 2, I32), full(rows, 0.99), full(rows, 0.0))
    assert torch.equal(token, allowed.int())


@pytest.mark.parametrize("vocab", [4, 64, 1024, 4096, 65536, 131072])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_logits_go_by_their_indices(vocab, dtype):
    """Weights of 1: every sum is exact, and u or p may meet a border."""
    rows = 9
    x = torch.full((rows, vocab), 2.5, device=DEV, dtype=dtype)
    u = torch.arange(rows, device=DEV) / 8.0
    token, logp = run(x, u)
    want = torch.clamp((u * vocab).floor(), max=vocab - 1).int()
    assert torch.equal(token, want) and bool((logp.double() + math.log(vocab)).abs().max() <= 1e-6)
    token, logp = run(x, u, None, full(rows, vocab // 2, I32))
    assert torch.equal(token, torch.clamp((u * (vocab // 2)).floor(), max=vocab // 2 - 1).int())
    token, logp = run(x, u, None, None, full(rows, 0.25))
    assert torch.equal(token, torch.clamp((u * (vocab // 4)).floor(), max=vocab // 4 - 1).int())
    token, logp = run(x, u, None, full(rows, vocab // 2, I32), full(rows, 0.5), full(rows, 1.0))
    assert torch.equal(token, torch.clamp((u * (vocab // 4)).floor(), max=vocab // 4 - 1).int())
    assert bool((logp.double() + math.log(vocab // 4)).abs().max() <= 1e-6)


@pytest.mark.parametrize("vocab", [40, 3000, 90000])
def test_ties_at_the_last_place(vocab):
    """Two values; the limits cut within the smaller one."""
    rows = 8
    x = torch.full((rows, vocab), 0.0, device=DEV, dtype=BF16)
    x[:, vocab // 3] = 1.0
    u = torch.linspace(0, 1, rows, device=DEV)
    for k in (1, 2, vocab // 2, vocab - 1):
        check(run(x, u, None, full(rows, k, I32)), x, u, None, full(rows, k, I32))
    for p in (0.001, 0.37, 0.5):
        check(run(x, u, None, None, full(rows, p)), x, u, None, None, full(rows, p))
        check(run(x, u, None, full(rows, vocab - 2, I32), full(rows, p)), x, u, None, full(rows, vocab - 2, I32), full(rows, p))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab,spread", [(8000, 1.0), (40000, 0.3), (128256, 0.5), (128256, 2.5)])
def test_limits_that_keep_few_many_and_most(vocab, spread, dtype):
    """What is kept is ranked, found in a list, or found in the row itself: from a few tokens to nearly all, by each limit and by two of them; with
    a share of banned tokens."""
    rows = 12
    x, u, *_ = make((rows, vocab, dtype, vocab, spread), seed=5)
    x = x.masked_fill(torch.rand((1, vocab), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 0.1, -math.inf)
    ks = torch.tensor([1, 7, 60, 250, 400, 700, 1500, 4000, 7000, vocab // 3, vocab - 5, vocab // 2], device=DEV, dtype=I32)
    ps = torch.tensor([0.001, 0.05, 0.2, 0.4, 0.6, 0.8, 0.9, 0.95, 0.99, 0.999, 0.99999, 0.5], device=DEV)
    qs = torch.tensor([0.9, 0.5, 0.2, 0.1, 0.05, 0.02, 0.01, 0.003, 1e-3, 1e-4, 1e-6, 1e-30], device=DEV)
    for limits in ((ks, None, None), (None, ps, None), (None, None, qs), (ks, ps.flip(0), None), (ks, None, qs.flip(0)), (None, ps, qs.flip(0)), (ks.flip(0), ps, qs)):
        check(run(x, u, None, *limits), x, u, None, *limits)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [9000, 50001, 140000])
def test_rows_in_order_and_in_steps(vocab, dtype):
    """The largest logits lie together, at either end or in the middle, or a few hundred of them are equal, where the limits keep thousands."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    z = torch.randn(vocab, generator=g, device=DEV).mul_(0.7).sort()[0]
    kinds = [z, z.flip(0), torch.roll(z, vocab // 2), (z[torch.randperm(vocab, generator=g, device=DEV)] * 64).round() / 64]
    limits = [(0, 0.5, 0.0), (0, 0.97, 0.0), (0, 0.999999, 0.0), (0, 0.97, 0.2), (vocab // 3, 1.0, 0.0), (vocab // 2, 0.9, 0.0), (vocab // 2, 0.9, 0.3), (0, 1.0, 0.1), (700, 0.9, 0.0)]
    rows = len(kinds) * len(limits)
    x = torch.stack([kinds[i // len(limits)] for i in range(rows)]).to(dtype)
    pick = lambda at, t=F32: torch.tensor([limits[i % len(limits)][at] for i in range(rows)], device=DEV, dtype=t)
    args = torch.rand(rows, generator=g, device=DEV), full(rows, 0.8), pick(0, I32), pick(1), pick(2)
    check(run(x, *args), x, *args)


@pytest.mark.parametrize("vocab", [50, 5000, 100000])
def test_logits_that_differ_in_their_last_bits(vocab):
    """fp32 logits closer to each other than their distance from the maximum can tell; and far apart."""
    rows = 6
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = torch.full((rows, vocab), 1.0, device=DEV) + torch.randint(0, 60, (rows, vocab), generator=g, device=DEV) * 2.0 ** -23
    x[:, 7] = 100.0
    x[3:] = torch.randn((3, vocab), generator=g, device=DEV) * torch.tensor([[1e4], [1e-30], [1e30]], device=DEV)
    u, k = torch.rand(rows, generator=g, device=DEV), full(rows, vocab // 2, I32)
    scale = torch.tensor([2.0 ** -6, 0.03, 1.0, 1e-4, 2.0 ** 60, 2.0 ** -60], device=DEV)
    for limits in ((scale, k, None, None), (scale, None, full(rows, 0.7), None), (scale, k, full(rows, 0.7), None)):
        check(run(x, u, *limits), x, u, *limits)


def far_above(rows, vocab, dtype, seed):
    """Rows whose logits lie 0 to 40 of the type's steps below a maximum that several share, the rest far below it or banned."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    top = torch.tensor([3.0, 10.0, 20.0, 100.0, 600.0, 1000.0, 0.0, -7.0, -0.001, -2000.0], device=DEV)[torch.arange(rows, device=DEV) % 10][:, None]
    steps = torch.randint(0, 41, (rows, vocab), generator=g, device=DEV) * torch.randint(0, 2, (rows, vocab), generator=g, device=DEV)
    size = torch.where(top == 0, 2.0 ** -149, torch.exp2(torch.floor(torch.log2(top.abs())))) * torch.finfo(dtype).eps
    x = top.double() - steps * size.double()
    kind = torch.rand((rows, vocab), generator=g, device=DEV)
    x = torch.where(kind < 0.5, top.double() - 1.0 - 50.0 * torch.rand((rows, vocab), generator=g, device=DEV), x)
    x = torch.where(kind < 0.2, -math.inf, x)
    few = torch.arange(rows, device=DEV) % 3 == 0  # the maximum once, near the end
    x = torch.where(few[:, None] & (x >= top), -math.inf, x)
    x[:, vocab - 2 if vocab > 2 else 0] = top[:, 0].double()
    return x.to(dtype), torch.rand(rows, generator=g, device=DEV)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [7, 300, 5000, 9000, 128256])
def test_scales_at_which_a_step_of_the_largest_logit_is_many_nats(vocab, dtype):
    """A tiny temperature: the numbers next to the largest logit weigh something, nothing, or less than 64 bits hold; with and without limits."""
    scales = [1e6, 2e6, 2.0 ** 24, 2.0 ** 27, 1e8, 2.0 ** 28, 1e9, 2.0 ** 30, 1e10, 2.0 ** 35, 2.0 ** 40, 2.0 ** 60, 1e3, 1e4, 1e5, 3e5]
    rows = 10 * len(scales)
    x, u = far_above(rows, vocab, dtype, seed=vocab)
    scale = torch.tensor(scales, device=DEV).repeat_interleave(10)
    k, p, q = full(rows, max(2, vocab // 9), I32), full(rows, 0.83), full(rows, 0.01)
    for limits in ((None, None, None), (None, None, q), (None, p, None), (k, None, None), (k, p, None), (k, p, q)):
        check(run(x, u, scale, *limits), x, u, scale, *limits)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [6, 700, 9000, 70000])
def test_rows_of_the_lowest_number(vocab, dtype):
    """Nothing is below the largest logit but what is banned, which weighs nothing all the same."""
    rows = 8
    x = torch.full((rows, vocab), torch.finfo(dtype).min, device=DEV, dtype=dtype)
    x[:, ::3] = -math.inf
    u = torch.linspace(0.03, 0.97, rows, device=DEV)
    for scale in (1.0, 2.0 ** -60, 2.0 ** 60):
        for limits in ((None, None, None), (full(rows, 3, I32), full(rows, 0.9), None), (None, full(rows, 0.6), full(rows, 0.2))):
            check(run(x, u, full(rows, scale), *limits), x, u, full(rows, scale), *limits)


def tail(n, x, scale, p, k):
    """One token of weight 1 and n[0], n[1] of logits x[0] > x[1]: how many of the latter top-p keeps of the first k, as a number whose next whole one it is."""
    w = [math.exp(scale * v) for v in x]
    n = [min(n[0], k - 1), min(n[1], max(0, k - 1 - n[0]))]
    left = (1.0 - p) * (1.0 + n[0] * w[0] + n[1] * w[1])  # what may be left out (1 - p is exact)
    first = n[1] - left / w[1]
    return n[0] + first if first > 0 else n[0] - (left - n[1] * w[1]) / w[0]


@pytest.mark.parametrize("vocab,dtype,n", [(4096, F32, 2000), (8192, BF16, 4000), (50257, F32, 20000), (128256, BF16, 5000), (128256, F16, 60000), (1048571, BF16, 500000)],
                         ids=lambda v: str(v))
def test_top_p_next_to_one_over_many_equal_logits_that_weigh_little(vocab, dtype, n):
    """What top-p leaves out are some of two kinds of equal logits of 2^-35 to 2^-43 each: a sum that loses a part of each of them ends elsewhere.  The
    number that is kept follows from the definition, and is never within a tenth of a whole one.  A thread adds vocab / 512 weights one after the other,
    one of which may be the 1: a sum is off by vocab / 512 2^-53 of the whole at most, which is less than a tenth of a token but in the longest row,
    where tokens of 2^-43 are two of them apart."""
    x, rows = (-28.0, -28.125), []
    for steps in (1, 2, 3):
        p = 1.0 - steps * 2.0 ** -24
        for offset in (-5.5, -1.5, -0.5, 0.5, 4.5, 0.4 * n):  # tokens beyond those of the first kind
            for k in (0, 1 + 2 * n - n // 3):
                count = k if k else vocab
                low, high = 0.5, 3.0  # the more scale, the fewer are kept
                for _ in range(80):
                    scale = 0.5 * (low + high)
                    low, high = (scale, high) if tail((n, n), x, scale, p, count) > n + offset else (low, scale)
                scale = torch.tensor(scale)
                kept = tail((n, n), x, float(scale), p, count)
                while not 0.1 < kept % 1.0 < 0.9:
                    scale = torch.nextafter(scale, torch.tensor(0.0))
                    kept = tail((n, n), x, float(scale), p, count)
                rows.append((p, float(scale), k, math.ceil(kept)))
    off = torch.tensor([math.ceil(max(0.0, vocab * 2.0 ** -62 / math.exp(r[1] * x[1]) - 0.1)) for r in rows], device=DEV)
    assert vocab > 1 << 18 or int(off.max()) == 0
    values = torch.full((2, vocab), -math.inf, device=DEV)
    values[0, 0], values[0, 1:n + 1], values[0, n + 1:2 * n + 1] = 0.0, x[0], x[1]
    values[1, vocab - 1], values[1, 7:n + 7], values[1, n + 7:2 * n + 7] = 0.0, x[1], x[0]
    pick = lambda at, t=F32: torch.tensor([r[at] for r in rows], device=DEV, dtype=t)
    p, scale, k, want = pick(0), pick(1), pick(2, I32), pick(3, I32)
    logits = values[0].to(dtype).expand(len(rows), vocab).contiguous()
    for limits in ((k, p, None), (k, p, full(len(rows), 1e-30))):
        token, logp = run(logits, full(len(rows), 1.0), scale, *limits)  # the last one that is kept
        assert bool(((token - want).abs() <= off).all()), (token - want).tolist()
        assert bool(((logp.double() - torch.where(want > n, x[1], x[0]) * scale.double()).abs() <= 30 * 2.0 ** -23).all())
    logits = values[1].to(dtype).expand(len(rows), vocab).contiguous()
    token, _ = run(logits, full(len(rows), 0.0), scale, k, p)  # the first one: of the second kind where any of them is kept
    assert bool((((want - n).abs() <= off) & (off > 0) | (token == torch.where(want > n, 7, n + 7))).all())


@pytest.mark.parametrize("vocab,dtype,n", [(4096, F32, 900), (8192, BF16, 1000), (4096, F32, 2000), (8192, F16, 4000), (20000, BF16, 4000), (9000, F32, 4400)],
                         ids=lambda v: str(v))
def test_top_p_a_small_part_of_a_token_from_the_end_of_equal_logits(vocab, dtype, n):
    """As above, with fewer tokens: the border is a small part of a token before or behind the last one of the first kind, where sums of weights rounded to
    2^-shift end on its other side in some rows.  (The parts are four times what sums may be off or more.)"""
    x, rows, missed = (-28.0, -28.125), [], 0
    unit = 2.0 ** min(50, 61 - (vocab - 1).bit_length())
    for steps in range(1, 13):
        p = 1.0 - steps * 2.0 ** -24
        for before in (True, False):
            low, high = 0.5, 3.0
            for _ in range(80):
                scale = 0.5 * (low + high)
                low, high = (scale, high) if tail((n, n), x, scale, p, vocab) > n else (low, scale)
            scale = torch.tensor(scale)
            part = 0.1 * min(1.0, n * unit ** -1 / math.exp(float(scale) * x[0]) * 4)
            for _ in range(1000):
                kept = tail((n, n), x, float(scale), p, vocab) - n
                if part / 5 < (-kept if before else kept) < part:
                    break
                scale = torch.nextafter(scale, torch.tensor(0.0 if kept < (-0.6 if before else 0.6) * part else 9.0))
            else:
                continue
            w, whole = [math.exp(float(scale) * v) for v in x], 1.0
            whole += n * w[0] + n * w[1]
            missed += (unit + n * round(w[0] * unit) >= round(p * whole * unit)) != before
            assert vocab * 2.0 ** -62 < part / 20 * w[1]
            rows.append((p, float(scale), n if before else n + 1))
    assert len(rows) >= 6 and missed >= 2, (len(rows), missed)
    values = torch.full((vocab,), -math.inf, device=DEV)
    values[0], values[1:n + 1], values[n + 1:2 * n + 1] = 0.0, x[0], x[1]
    pick = lambda at, t=F32: torch.tensor([r[at] for r in rows], device=DEV, dtype=t)
    logits = values.to(dtype).expand(len(rows), vocab).contiguous()
    token, _ = run(logits, full(len(rows), 1.0), pick(1), None, pick(0))
    assert torch.equal(token, pick(2, I32)), (token - pick(2, I32)).tolist()


def test_every_token_comes_as_often_as_it_should():
    vocab, rows = 10, 4096
    row = torch.randn(vocab, device=DEV)
    u = (torch.arange(rows, device=DEV) + 0.5) / rows
    token, logp = run(row.expand(rows, vocab).contiguous(), u)
    p = torch.softmax(row.double(), 0)
    assert bool(((torch.bincount(token.long(), minlength=vocab) / rows - p).abs() <= 2 / rows).all())
    assert bool((logp.double() - torch.log(p)[token.long()]).abs().max() <= 1e-6)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_unaligned_rows_other_streams_and_graphs(dtype):
    rows, vocab = 21, 9001
    space = torch.randn(rows * 9003 + 1, device=DEV).to(dtype)
    x = torch.as_strided(space, (rows, vocab), (9003, 1), 1)
    _, u, scale, k, p, q = make((rows, vocab, dtype, vocab, 1.0))
    d = lib.sm_desc_create(lib.SmParams(rows, vocab, dtype))
    ws = torch.empty(lib.sm_desc_workspace_bytes(d) // 4 + 1, device=DEV)
    token, logp = torch.empty(rows, device=DEV, dtype=I32), torch.empty(rows, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lib.sm_sample(d, x, u, scale, k, p, q, token, logp, ws, side)
    side.synchronize()
    check((token, logp), x, u, scale, k, p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.sm_sample(d, x, u, scale, k, p, q, token, logp, ws)
    for _ in range(3):
        space.normal_()
        u.uniform_()
        k.copy_(k.roll(1))
        graph.replay()
        replayed = token.clone()
        lib.sm_sample(d, x, u, scale, k, p, q, token, logp, ws)
        torch.cuda.synchronize()
        assert torch.equal(replayed, token)
        check((token, logp), x, u, scale, k, p, q)


def test_no_rows_and_far_rows():
    d = lib.sm_desc_create(lib.SmParams(0, 100, F32))
    lib.sm_sample(d, torch.empty((0, 100), device=DEV), torch.empty(0, device=DEV), None, None, None, None, torch.empty(0, device=DEV, dtype=I32))
    x = torch.empty((2, 5000), device=DEV, dtype=BF16)  # rows more than 2^32 bytes apart
    space = torch.zeros((1 << 31) + 6000, device=DEV, dtype=BF16)
    far = torch.as_strided(space, (2, 5000), ((1 << 31) + 500, 1))
    far[0, 11], far[1, 4999] = 50.0, 50.0
    token, _ = run(far, full(2, 0.5))
    assert token.tolist() == [11, 4999]


def test_more_rows_than_a_launch_has_workgroups():
    rows, vocab = (1 << 20) + 5, 3
    x = torch.randn((1000, vocab), device=DEV).repeat(-(-rows // 1000), 1)[:rows].contiguous()
    u = torch.rand(1000, device=DEV).repeat(-(-rows // 1000))[:rows].contiguous()
    for limits in ((None, None, None, None), (None, full(rows, 2, I32), full(rows, 0.9), None)):
        token, logp = run(x, u, *limits)
        check((token[:1000], logp[:1000]), x[:1000], u[:1000], *(None if t is None else t[:1000] for t in limits))
        assert torch.equal(token, token[:1000].repeat(-(-rows // 1000))[:rows])

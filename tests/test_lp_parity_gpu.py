"""Log probabilities of given tokens, entropy, alternatives and gradients (include/mi355lp.h) against the oracle in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32): a row's sum is at most 256 additions deep in these sizes (per thread, then over lanes,
waves and parts), each term 2^t has its exponent rounded once (|t| u) and a table's error of 2 u.
  log p     256 u + 4 u |log p|
  entropy   256 u (2 + log2 vocab): s2 / s and log2 s, each off by the sums' error
  gradient  u (300 + 2 |t|) on each of its terms, p |w| and p |u| (|log p| + H + 2 log2 vocab) (the constants' cancellation), two
            roundings of w at the token, then half a step of the output's type, or of its smallest number
"""
import math

import pytest
import torch

import paper_1810_02272_amd as lib
from oracle import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = 2.0 ** -24
INF = math.inf

# rows, vocab, dtype, top, entropy, scale, gap between rows, first element's place in its buffer
CASES = [
    (1, 1, F32, 1, 1, 1.0, 0, 0),
    (3, 2, BF16, 2, 1, 1.0, 0, 1),
    (5, 7, F16, 3, 1, 0.5, 0, 1),
    (4, 8, BF16, 8, 0, 1.0, 1, 0),
    (9, 9, BF16, 1, 1, 2.0, 0, 3),
    (6, 31, F32, 31, 1, 1.0, 2, 1),
    (7, 64, F16, 64, 1, 1.0, 0, 0),
    (300, 65, BF16, 20, 1, 1.0, 0, 0),
    (17, 511, F32, 32, 1, 1.5, 0, 0),
    (33, 1000, F32, 0, 0, 1.0, 0, 0),
    (5, 1024, F32, 5, 1, 1.0, 0, 0),
    (5, 1025, F32, 5, 1, 1.0, 0, 3),
    (5, 2048, BF16, 5, 1, 1.0, 0, 0),
    (2100, 333, F16, 7, 1, 1.0, 5, 0),       # several rows in a workgroup
    (5, 2049, F16, 40, 1, 0.75, 0, 0),
    (11, 5000, BF16, 64, 1, 1.0, 8, 0),
    (270, 8190, F32, 10, 1, 1.0, 2, 2),
    (260, 16384, BF16, 20, 1, 1.0, 0, 0),
    (300, 9001, F16, 20, 1, 1.0, 0, 3),
    (300, 2050, BF16, 20, 1, 1.0, 0, 0),
    (2049, 4096, F16, 20, 1, 1.0, 1, 1),
    (300, 1999, F32, 20, 1, 1.0, 0, 0),
    (300, 32768, BF16, 20, 1, 1.0, 0, 0),
    (300, 9000, F32, 20, 1, 1.0, 0, 2),
    (600, 40001, F16, 20, 1, 1.0, 0, 0),
    (600, 26624, F32, 64, 1, 1.0, 0, 0),
    (300, 90003, F16, 64, 1, 1.0, 0, 1),
    (257, 16387, F16, 20, 0, 1.0, 0, 5),
    (256, 32768, F32, 3, 1, 1.0, 0, 0),
    (520, 50257, BF16, 20, 1, 1.25, 47, 0),
    (256, 65539, F16, 32, 1, 1.0, 0, 0),
    (256, 90001, F32, 20, 1, 1.0, 0, 0),     # beyond a workgroup's registers
    (256, 128256, BF16, 20, 1, 1.0, 0, 0),
    (256, 163900, BF16, 5, 0, 1.0, 0, 0),    # beyond a workgroup's registers
    (1, 8192, BF16, 20, 1, 1.0, 0, 0),       # a row in parts
    (1, 32000, BF16, 20, 1, 1.0, 0, 0),
    (2, 10001, F32, 64, 1, 1.0, 3, 1),
    (3, 160000, F16, 20, 1, 1.0, 0, 0),
    (64, 50257, BF16, 20, 1, 1.5, 0, 0),
    (130, 20011, F32, 32, 1, 1.0, 1, 0),
    (1, 128257, BF16, 64, 1, 1.0, 0, 1),
    (4, 40009, F32, 20, 1, 0.5, 3, 0),
    (128, 33000, F16, 20, 1, 1.0, 0, 0),
    (20, 16385, F32, 20, 1, 1.0, 0, 0),
    (1, 1000000, F16, 20, 1, 1.0, 0, 0),
    (70001, 2000, BF16, 3, 1, 1.0, 0, 0),    # more than the last-level cache holds
    (20001, 8001, BF16, 3, 1, 1.0, 0, 0),
    (40001, 3999, BF16, 3, 1, 1.0, 0, 0),
    (6001, 30001, BF16, 3, 1, 1.0, 0, 0),
    (3001, 50257, BF16, 3, 1, 1.0, 0, 0),
    (1100, 128256, BF16, 20, 1, 1.0, 0, 0),
]
IDS = ["%dx%d-%s-t%d-e%d-s%g-g%d-o%d" % (c[0], c[1], str(c[2])[6:], *c[3:]) for c in CASES]


def spaced(values, dtype, gap, first):
    """The rows in a buffer of their own with a gap behind each, and the buffer (NaN where no element is)."""
    rows, vocab = values.shape
    buffer = torch.full((first + rows * (vocab + gap) + 8,), math.nan, device=DEV, dtype=dtype)
    view = buffer[first:first + rows * (vocab + gap)].view(rows, vocab + gap)[:, :vocab]
    view.copy_(values)
    return view, buffer


def untouched(view, buffer):
    """Whether the buffer still holds NaN wherever the view has no element."""
    rest = torch.ones_like(buffer, dtype=torch.bool)
    rest.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool(torch.isnan(buffer[rest]).all())


def make(case, seed):
    rows, vocab, dtype, top, entropy, scale, gap, first = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g, device=DEV) * 2.5
    if vocab > 20:
        x.masked_fill_(torch.rand((1, vocab), generator=g, device=DEV) < 0.05, -INF)
    token = torch.randint(vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if rows > 4:  # rows at which it can go wrong
        x[1] = -INF                                             # nothing left
        x[2] = torch.finfo(dtype).min                           # the type's lowest value throughout
        x[3] = -INF
        x[3, vocab // 2] = -3.0                                 # one left, and another is asked for
        x[4] = 0.25                                             # equal throughout
        token[0], token[3] = -1, 0
    if rows > 8:
        x[5] = torch.finfo(dtype).min
        x[5, vocab - 1] = 2.0
        x[6, ::2] = 0.0
        x[6, 1::2] = -0.0
        x[7] = torch.linspace(-9, 9, vocab, device=DEV)         # the likeliest next to each other
        token[6], token[7] = vocab, 2 ** 31 - 1
    if rows > 16:
        x[9] = torch.linspace(9, -9, vocab, device=DEV)
        x[10] = -1000.0 + 0.01 * torch.arange(vocab, device=DEV) % 64
        x[11] += 500.0
    x, buffer = spaced(x.to(dtype), dtype, gap, first)
    d_logp = torch.randn(rows, generator=g, device=DEV)
    d_entropy = torch.randn(rows, generator=g, device=DEV) * 0.1 if entropy else None
    return x, buffer, token, d_logp, d_entropy


def within(got, want, tol, what):
    got, want = got.double(), want.double()
    same = (got == want.to(torch.float32)) | ((got - want).abs() <= tol)  # (what fp32 does not reach is an infinity)
    assert bool(same.all()), (what, float(torch.where(same, 0.0, (got - want).abs()).nan_to_num(INF).max()), int((~same).sum()))


def check_rows(logp, h, got_logp, got_h, token, vocab):
    within(got_logp, tokens.token_logp(logp, token), U * (256 + 4 * tokens.token_logp(logp, token).abs().nan_to_num(0, 0, 0)), "logp")
    if got_h is not None:
        within(got_h, h, U * 256 * (2 + math.log2(vocab)), "entropy")


def check_gradient(case, x, token, d_logp, d_entropy, got):
    rows, vocab, dtype, _, _, scale, _, _ = case
    logp, h = tokens.log_probs(x, scale)
    p = logp.exp()
    valid = (token >= 0) & (token < vocab)
    w = torch.where(valid, d_logp.double(), 0.0).abs()[:, None]
    inner = torch.where(p == 0, torch.zeros_like(p), p * (logp.abs() + h[:, None] + 2 * math.log2(vocab)))
    depth = 300 + 2 * logp.abs().clamp(max=200) * 1.5
    tol = scale * U * depth * (p * w + (inner * d_entropy.double().abs()[:, None] if d_entropy is not None else 0.0))
    at = torch.where(valid, token, 0).long()[:, None]
    tol.scatter_add_(1, at, torch.where(valid[:, None], 2 * U * scale * w, 0.0))
    want = tokens.d_logits(x, token, d_logp, d_entropy, scale)
    info = torch.finfo(dtype)
    tol += want.abs() * (info.eps / 2) + (2.0 ** -25 if dtype == F16 else 2.0 ** -126)
    within(got, want, tol, "d_logits")


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_parity(case):
    rows, vocab, dtype, top, entropy, scale, gap, first = case
    x, x_buffer, token, d_logp, d_entropy = make(case, seed=rows * 7 + vocab)
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, dtype, top, entropy, scale))
    print(lib.lp_desc_kernel_names(d), flush=True)
    ws_bytes = lib.lp_desc_workspace_bytes(d)
    ws = torch.full((ws_bytes // 4 + 64,), math.nan, device=DEV)
    nan = lambda *shape: torch.full(shape, math.nan, device=DEV)
    logp, h, stats = nan(rows), nan(rows) if entropy else None, nan(rows, 4)
    top_logp = nan(rows, top) if top else None
    top_token = torch.full((rows, top), -7, device=DEV, dtype=torch.int32) if top else None
    lib.lp_forward(d, x, token, logp, h, stats, top_logp, top_token, ws[:(ws_bytes + 3) // 4])
    assert torch.isnan(ws[(ws_bytes + 3) // 4:]).all()
    want_logp, want_h = tokens.log_probs(x, scale)
    check_rows(want_logp, want_h, logp, h, token, vocab)
    if top:
        index = tokens.top_tokens(x, top)
        assert torch.equal(top_token.long(), index)
        want = want_logp.gather(1, index)
        within(top_logp, want, U * (256 + 4 * want.abs().nan_to_num(0, 0, 0)), "top_logp")

    g, g_buffer = spaced(nan(rows, vocab), dtype, gap // 2, (first + 1) % 4)
    lib.lp_backward(d, x, token, stats, d_logp, d_entropy, g)
    check_gradient(case, x, token, d_logp, d_entropy, g)
    assert untouched(g, g_buffer)

    g2, g2_buffer = spaced(nan(rows, vocab), dtype, gap, first)
    logp2, h2 = nan(rows), nan(rows) if entropy else None
    lib.lp_forward_backward(d, x, token, d_logp, d_entropy, logp2, h2, g2, ws)
    check_rows(want_logp, want_h, logp2, h2, token, vocab)
    check_gradient(case, x, token, d_logp, d_entropy, g2)
    assert untouched(g2, g2_buffer)

    # equal calls, equal bits; what is not wanted is left out
    g3 = torch.empty_like(g2)
    lib.lp_forward_backward(d, x, token, d_logp, d_entropy, None, None, g3, ws)
    assert torch.equal(g3, g2)
    # in place
    before = x.clone()
    lib.lp_forward_backward(d, x, token, d_logp, d_entropy, logp2, h2, x, ws)
    assert torch.equal(x, g2) and untouched(x, x_buffer)
    check_rows(want_logp, want_h, logp2, h2, token, vocab)
    x.copy_(before)
    lib.lp_backward(d, x, token, stats, d_logp, d_entropy, x)
    assert torch.equal(x, g) and untouched(x, x_buffer)


@pytest.mark.parametrize("scale", [1.0, 1.5, 0.37, 2.0 ** 20])
@pytest.mark.parametrize("vocab", [500, 3000, 9001, 40000, 70001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_finite_logits(dtype, vocab, scale):
    """Masks of -1e9 and on, throughout a row, in a run that some threads see nothing but, and next to each other; large positive
    logits; differences of one step of the type at either end of the range."""
    rows = 24
    x = torch.randn((rows, vocab), device=DEV) * 2
    for r, mask in enumerate((-1e9, -1e10, -3e15, -1e20, -1e30, -3e38)):
        x[r] = mask                                  # throughout
        x[6 + r] = mask
        x[6 + r, -3:] = torch.tensor([1.0, 2.0, 0.5], device=DEV)  # all but three
        x[12 + r, : vocab // 2] = mask               # half
    x[18] = 1e9
    x[18, 7] = 1.1e9
    x[19, 3] = 3e38
    x[20] = -1e30
    x[20, : vocab // 3] = -1.01e30
    x[21] *= 1e8
    x[22] = -3e8
    x = x.to(dtype)
    x[23] = -1e25
    x[23, 5] = torch.nextafter(x[23, 5].cpu(), torch.tensor(0.0, dtype=dtype)).to(DEV)
    token = torch.randint(vocab, (rows,), device=DEV, dtype=torch.int32)
    token[18], token[23] = 7, 5
    w, u = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV) * 0.1
    want_logp, want_h = tokens.log_probs(x, scale)
    case = (rows, vocab, dtype, 5, 1, scale, 0, 0)
    for copies in (1, 30):  # 30: teams of rows that many
        n = rows * copies
        many = x.repeat(copies, 1)
        d = lib.lp_desc_create(lib.LpParams(n, vocab, dtype, 5, 1, scale))
        print(lib.lp_desc_kernel_names(d), flush=True)
        ws = torch.empty(lib.lp_desc_workspace_bytes(d) // 4 + 1, device=DEV)
        logp, h, stats = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty((n, 4), device=DEV)
        tl, tt = torch.empty((n, 5), device=DEV), torch.empty((n, 5), device=DEV, dtype=torch.int32)
        lib.lp_forward(d, many, token.repeat(copies), logp, h, stats, tl, tt, ws)
        g, g2, logp2, h2 = torch.empty_like(many), torch.empty_like(many), torch.empty_like(logp), torch.empty_like(h)
        lib.lp_backward(d, many, token.repeat(copies), stats, w.repeat(copies), u.repeat(copies), g)
        lib.lp_forward_backward(d, many, token.repeat(copies), w.repeat(copies), u.repeat(copies), logp2, h2, g2, ws)
        for at in (slice(0, rows), slice(n - rows, n)):
            check_rows(want_logp, want_h, logp[at], h[at], token, vocab)
            check_rows(want_logp, want_h, logp2[at], h2[at], token, vocab)
            index = tokens.top_tokens(x, 5)
            assert torch.equal(tt[at].long(), index)
            want = want_logp.gather(1, index)
            within(tl[at], want, U * (256 + 4 * want.abs()), "top_logp")
            check_gradient(case, x, token, w, u, g[at])
            check_gradient(case, x, token, w, u, g2[at])


@pytest.mark.parametrize("rows,vocab,dtype", [(6, 300, BF16), (6, 9000, F32), (6, 3000, F16), (260, 17000, BF16), (256, 100000, F32), (300, 3000, F16),
                                              (300, 8000, BF16), (600, 40000, BF16), (6, 70000, BF16)])
def test_not_a_number_and_infinity_reach_the_whole_row_and_no_other(rows, vocab, dtype):
    x = torch.randn((rows, vocab), device=DEV).to(dtype)
    x[1, vocab // 3] = math.nan
    x[2, vocab - 1] = INF
    x[3] = math.nan
    x[4, 0], x[4, 1:] = -math.nan, -INF
    token = torch.zeros(rows, dtype=torch.int32, device=DEV)
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, dtype, 4, 1))
    ws = torch.empty(lib.lp_desc_workspace_bytes(d) // 4 + 1, device=DEV)
    logp, h, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV)
    tl, tt = torch.empty((rows, 4), device=DEV), torch.empty((rows, 4), device=DEV, dtype=torch.int32)
    lib.lp_forward(d, x, token, logp, h, stats, tl, tt, ws)
    bad = [1, 2, 3, 4]
    good = [0] + list(range(5, rows))
    assert torch.isnan(logp[bad]).all() and torch.isnan(h[bad]).all() and torch.isnan(tl[bad]).all()
    assert torch.isfinite(logp[good]).all() and torch.isfinite(h[good]).all() and torch.isfinite(tl[good]).all()
    assert torch.equal(tt.long(), tokens.top_tokens(x, 4))
    w = torch.ones(rows, device=DEV)
    g, g2 = torch.empty_like(x), torch.empty_like(x)
    lib.lp_backward(d, x, token, stats, w, w, g)
    lib.lp_forward_backward(d, x, token, w, w, logp, h, g2, ws)
    for t in (g, g2):
        assert torch.isnan(t[bad]).all() and torch.isfinite(t[good]).all()


def test_gradient_against_differences():
    """Central differences of logp and entropy as the library itself gives them, fp32: a step of 2^-6 leaves h^2 / 6 of a third
    derivative that is at most 2 (4e-5 of |w| + |u|), and the values' own error over the step, 2^-24 600 / 2^-6 (2.3e-3 for these sizes)."""
    rows, vocab, step = 8, 40, 2.0 ** -6
    x = torch.randn((rows, vocab), device=DEV)
    token = torch.arange(rows, device=DEV, dtype=torch.int32)
    w, u = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV)
    one = lib.lp_desc_create(lib.LpParams(rows, vocab, F32, 0, 1))
    g = torch.empty_like(x)
    lib.lp_forward_backward(one, x, token, w, u, None, None, g)
    many = lib.lp_desc_create(lib.LpParams(rows * vocab, vocab, F32, 0, 1))

    def loss(sign):
        moved = x.repeat_interleave(vocab, 0) + sign * step * torch.eye(vocab, device=DEV).repeat(rows, 1)
        logp, h = torch.empty(rows * vocab, device=DEV), torch.empty(rows * vocab, device=DEV)
        lib.lp_forward(many, moved, token.repeat_interleave(vocab), logp, h)
        return (logp.double().view(rows, vocab) * w[:, None] + h.double().view(rows, vocab) * u[:, None])

    difference = (loss(1) - loss(-1)) / (2 * step)
    assert float((difference - g.double()).abs().max()) < 3e-3 * float(w.abs().max() + u.abs().max())


def test_more_rows_than_teams():
    rows, vocab = (1 << 22) + 77, 9  # four to a workgroup, 2^20 workgroups
    x = torch.randn((rows, vocab), device=DEV).to(BF16)
    token = torch.randint(vocab, (rows,), device=DEV, dtype=torch.int32)
    w, u = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV)
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, BF16, 2, 1))
    logp, h, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV)
    tl, tt = torch.empty((rows, 2), device=DEV), torch.empty((rows, 2), device=DEV, dtype=torch.int32)
    lib.lp_forward(d, x, token, logp, h, stats, tl, tt)
    check_rows(*tokens.log_probs(x), logp, h, token, vocab)
    assert torch.equal(tt.long(), tokens.top_tokens(x, 2))
    case = (rows, vocab, BF16, 2, 1, 1.0, 0, 0)
    g = torch.empty_like(x)
    lib.lp_backward(d, x, token, stats, w, u, g)
    check_gradient(case, x, token, w, u, g)
    g.fill_(math.nan)
    lib.lp_forward_backward(d, x, token, w, u, logp, h, g)
    check_gradient(case, x, token, w, u, g)


def test_far_rows():
    """Rows whose offset passes 2^31 elements."""
    vocab, stride, rows = 500, (1 << 30) + 24, 3
    buffer = torch.empty(stride * (rows - 1) + vocab, device=DEV, dtype=BF16)
    x = buffer.as_strided((rows, vocab), (stride, 1))
    x.copy_(torch.randn((rows, vocab), device=DEV))
    token = torch.tensor([3, 499, 7], device=DEV, dtype=torch.int32)
    w = torch.ones(rows, device=DEV)
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, BF16, 3, 1))
    logp, h, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV)
    tl, tt = torch.empty((rows, 3), device=DEV), torch.empty((rows, 3), device=DEV, dtype=torch.int32)
    lib.lp_forward(d, x, token, logp, h, stats, tl, tt)
    check_rows(*tokens.log_probs(x), logp, h, token, vocab)
    assert torch.equal(tt.long(), tokens.top_tokens(x, 3))
    case = (rows, vocab, BF16, 3, 1, 1.0, 0, 0)
    before = x.clone()
    lib.lp_backward(d, x, token, stats, w, None, x)
    check_gradient(case, before, token, w, None, x)
    x.copy_(before)
    lib.lp_forward_backward(d, x, token, w, w, None, None, x)
    check_gradient(case, before, token, w, w, x)


@pytest.mark.parametrize("rows,vocab", [(300, 1000), (3, 40000)])
def test_on_another_stream_and_in_a_graph(rows, vocab):
    """Captured once; replayed with new inputs, eager calls of the same buffers in between."""
    case = (rows, vocab, BF16, 5, 1, 1.0, 0, 0)
    x, _, token, w, u = make(case, seed=1)
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, BF16, 5, 1))
    ws = torch.empty(lib.lp_desc_workspace_bytes(d) // 4 + 1, device=DEV)
    logp, h = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    tl, tt = torch.empty((rows, 5), device=DEV), torch.empty((rows, 5), device=DEV, dtype=torch.int32)
    g = torch.empty_like(x)

    def step(stream=None):
        lib.lp_forward(d, x, token, logp, h, None, tl, tt, ws, stream)
        lib.lp_forward_backward(d, x, token, w, u, None, None, g, ws, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    first = [t.clone() for t in (logp, h, tl, tt, g)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3, 4):
        x.copy_(make(case, seed)[0])
        graph.replay()
        replayed = [t.clone() for t in (logp, h, tl, tt, g)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (logp, h, tl, tt, g)))
    x.copy_(make(case, 1)[0])
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(first, (logp, h, tl, tt, g)))


def test_refusals_on_the_device():
    d = lib.lp_desc_create(lib.LpParams(4, 90000, BF16, 2, 1))
    x = torch.zeros((4, 90000), device=DEV, dtype=BF16)
    token = torch.zeros(4, device=DEV, dtype=torch.int32)
    f = lambda *s: torch.empty(s, device=DEV)
    tl, tt, ws = f(4, 2), torch.empty((4, 2), device=DEV, dtype=torch.int32), f(lib.lp_desc_workspace_bytes(d) // 4)
    ok = lambda **k: lib.lp_forward(d, **{**dict(logits=x, token=token, logp=f(4), entropy=f(4), stats=None, top_logp=tl, top_token=tt, ws=ws), **k})
    ok()
    for wrong, error in ((dict(logits=x.float()), TypeError), (dict(logits=x.t()), ValueError), (dict(logits=x[:, :89999]), ValueError),
                         (dict(logits=torch.zeros((90000, 4), device=DEV, dtype=BF16).t()), TypeError),
                         (dict(logits=x[:1].expand(4, 90000)), TypeError), (dict(logits=x.cpu()), TypeError),
                         (dict(token=token.long()), TypeError), (dict(token=token[:3]), ValueError), (dict(logp=f(5)), ValueError),
                         (dict(token=None), lib.ConvError), (dict(top_logp=None), lib.ConvError), (dict(ws=None), lib.ConvError),
                         (dict(ws=ws[:-1]), lib.ConvError), (dict(stats=f(4, 3)), ValueError)):
        with pytest.raises(error):
            ok(**wrong)
    plain = lib.lp_desc_create(lib.LpParams(4, 90000, BF16, 0, 0))
    with pytest.raises(lib.ConvError):
        lib.lp_forward(plain, x, token, f(4), f(4), None, None, None, ws)
    with pytest.raises(lib.ConvError):
        lib.lp_backward(plain, x, token, f(4, 4), f(4), f(4), torch.empty_like(x))


def exponents_that_round_to(reference, scale, dtype):
    """Values of the type, next to each other, whose product with scale log2(e), as the kernels round it to fp32, is `reference`."""
    c = (torch.tensor(scale, dtype=F32).double() * 1.44269504088896340736).to(F32)
    x = torch.tensor(reference / float(c)).to(dtype)
    found = []
    for toward in (-INF, INF):
        at = x
        for _ in range(8):
            found.append(float(at))
            at = torch.nextafter(at, torch.tensor(toward, dtype=dtype))
    return sorted({v for v in found if float(torch.tensor(v, dtype=F32) * c) == reference})


@pytest.mark.parametrize("dtype,scale,vocab", [(F32, 1.0, 40000), (F32, 1.0, 17001), (F32, 0.37, 70001), (F32, 2.0 ** 20, 40000), (BF16, math.log(2), 70001),
                                               (BF16, 2.0 ** -40 * math.log(2), 40000), (BF16, 2.0 ** -40 * math.log(2), 128256)])
def test_largest_logit_at_the_end_of_the_references(dtype, scale, vocab):
    """Rows whose largest exponent is the least that a reference holds, -2^30, among masks beyond it: alone, several, in the first and the last
    part of a row, with masks one step of the type below; and rows of nothing but such masks."""
    best = exponents_that_round_to(-2.0 ** 30, scale, dtype)
    assert best
    below = float(torch.nextafter(torch.tensor(best[0], dtype=dtype), torch.tensor(-INF, dtype=dtype)))
    rows = 6 + len(best)
    x = torch.full((rows, vocab), -1e30, device=DEV)
    x[0, 0] = best[-1]
    x[1, vocab - 1] = best[-1]
    x[2, ::vocab // 3] = best[-1]
    x[3], x[3, vocab // 2] = below, best[-1]
    x[4] = below
    x[5, : vocab // 2], x[5, 7] = below, best[0]
    for r, value in enumerate(best):
        x[6 + r, 11 * r] = value
    x = x.to(dtype)
    token = torch.zeros(rows, device=DEV, dtype=torch.int32)
    token[1], token[5] = vocab - 1, 7
    want_logp, want_h = tokens.log_probs(x, scale)
    w, u = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV) * 0.1
    case = (rows, vocab, dtype, 5, 1, scale, 0, 0)
    for copies in (1, 50):  # rows in parts, and teams of a whole row
        n = rows * copies
        many, tokens_ = x.repeat(copies, 1), token.repeat(copies)
        d = lib.lp_desc_create(lib.LpParams(n, vocab, dtype, 5, 1, scale))
        print(lib.lp_desc_kernel_names(d), flush=True)
        ws = torch.empty(lib.lp_desc_workspace_bytes(d) // 4 + 1, device=DEV)
        logp, h, stats = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty((n, 4), device=DEV)
        tl, tt = torch.empty((n, 5), device=DEV), torch.empty((n, 5), device=DEV, dtype=torch.int32)
        lib.lp_forward(d, many, tokens_, logp, h, stats, tl, tt, ws)
        g, g2, logp2, h2 = torch.empty_like(many), torch.empty_like(many), torch.empty_like(logp), torch.empty_like(h)
        lib.lp_backward(d, many, tokens_, stats, w.repeat(copies), u.repeat(copies), g)
        lib.lp_forward_backward(d, many, tokens_, w.repeat(copies), u.repeat(copies), logp2, h2, g2, ws)
        for at in (slice(0, rows), slice(n - rows, n)):
            check_rows(want_logp, want_h, logp[at], h[at], token, vocab)
            check_rows(want_logp, want_h, logp2[at], h2[at], token, vocab)
            index = tokens.top_tokens(x, 5)
            assert torch.equal(tt[at].long(), index)
            want = want_logp.gather(1, index)
            within(tl[at], want, U * (256 + 4 * want.abs()), "top_logp")
            check_gradient(case, x, token, w, u, g[at])
            check_gradient(case, x, token, w, u, g2[at])


@pytest.mark.parametrize("rows,vocab,dtype", [(6, 300, BF16), (6, 9000, F32), (6, 3000, F16), (260, 17000, BF16), (256, 100000, F32), (300, 3000, F16),
                                              (300, 8000, BF16), (600, 40000, BF16), (6, 70000, BF16), (6, 17000, F32)])
def test_not_a_number_reaches_masked_tokens(rows, vocab, dtype):
    """Tokens and alternatives at masks of the type's lowest value, whose product with the scale leaves fp32, in rows with a NaN or +inf."""
    x = torch.randn((rows, vocab), device=DEV).to(dtype)
    lowest = torch.finfo(dtype).min
    for r, odd in ((1, math.nan), (2, INF), (3, math.nan)):
        x[r] = lowest
        x[r, vocab // 3] = odd
    x[1, 1] = 5.0
    token = torch.zeros(rows, dtype=torch.int32, device=DEV)
    token[1], token[2], token[3] = 2, vocab - 1, 0
    d = lib.lp_desc_create(lib.LpParams(rows, vocab, dtype, 4, 1))
    print(lib.lp_desc_kernel_names(d), flush=True)
    ws = torch.empty(lib.lp_desc_workspace_bytes(d) // 4 + 1, device=DEV)
    logp, logp2, h = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    tl, tt = torch.empty((rows, 4), device=DEV), torch.empty((rows, 4), device=DEV, dtype=torch.int32)
    lib.lp_forward(d, x, token, logp, h, None, tl, tt, ws)
    lib.lp_forward_backward(d, x, token, torch.ones(rows, device=DEV), None, logp2, None, torch.empty_like(x), ws)
    good = [0] + list(range(4, rows))
    for t in (logp, logp2, tl):
        assert torch.isnan(t[1:4]).all() and torch.isfinite(t[good]).all()
    assert torch.equal(tt.long(), tokens.top_tokens(x, 4))


@pytest.mark.parametrize("rows,vocab", [(40, 300), (3, 40000), (600, 30000)])
def test_statistics_without_entropy(rows, vocab):
    """By a descriptor without entropy: gradients through log p alone are right by either kind of descriptor, those through the entropy are NaN,
    not numbers of something else."""
    case = (rows, vocab, F32, 0, 1, 1.0, 0, 0)
    x, _, token, w, u = make(case, seed=4)
    plain, full = (lib.lp_desc_create(lib.LpParams(rows, vocab, F32, 0, e)) for e in (0, 1))
    ws = torch.empty(max(lib.lp_desc_workspace_bytes(d) for d in (plain, full)) // 4 + 1, device=DEV)
    logp, stats, g = torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV), torch.empty_like(x)
    lib.lp_forward(plain, x, token, logp, None, stats, None, None, ws)
    for d in (plain, full):
        g.fill_(math.nan)
        lib.lp_backward(d, x, token, stats, w, None, g)
        check_gradient(case, x, token, w, None, g)
    lib.lp_backward(full, x, token, stats, w, u, g)
    some = (x > -INF).sum(1) > 0  # (a row of nothing but -inf has no gradient through the entropy)
    assert torch.isnan(g[some]).all()
    lib.lp_forward(full, x, token, logp, None, stats, None, None, ws)
    lib.lp_backward(full, x, token, stats, w, u, g)
    check_gradient(case, x, token, w, u, g)

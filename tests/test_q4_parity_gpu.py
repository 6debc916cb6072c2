"""The InnerProduct layer on 4-bit weights (include/mi355q4.h) against the oracle in 64 bits.

Tolerance: products are exact, sums in fp32.  An output passes at most k / 128 + 4 additions of groups' sums (128 terms each, summed
by the matrix unit) and their joining, so its error is below (k / 32 + 160) 2^-24 of the sum of the terms' magnitudes, plus the bias's addition;
then half a step of the output's type, or of its smallest number."""
import math

import pytest
import torch

import paper_1810_02272_amd as lib
from oracle import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

# m, k, o, dtype, group, bias, relu
CASES = [
    (1, 1, 1, BF16, 32, 0, 0), (1, 32, 8, F32, 32, 1, 1), (2, 33, 17, F16, 32, 1, 0), (3, 127, 16, BF16, 64, 0, 1), (5, 128, 15, F32, 128, 1, 0),
    (1, 129, 31, BF16, 128, 0, 0), (4, 1000, 100, F16, 64, 1, 1), (1, 4096, 4096, BF16, 128, 0, 0), (1, 4095, 777, BF16, 32, 1, 0),
    (15, 2047, 65, F32, 64, 0, 0), (16, 2048, 64, BF16, 32, 0, 0), (17, 640, 300, F16, 128, 1, 1), (31, 999, 2000, BF16, 64, 1, 1),
    (33, 12288, 40, BF16, 64, 0, 0), (48, 9216, 256, F32, 64, 1, 1), (49, 500, 1111, F32, 32, 0, 0), (64, 1536, 512, F16, 32, 0, 1),
    (9, 700, 5000, BF16, 64, 1, 0), (12, 300, 6000, F32, 32, 0, 0), (7, 900, 5000, F32, 64, 1, 1), (58, 161, 3467, BF16, 64, 0, 0), (14, 4337, 1534, F16, 32, 0, 1),
    (9, 2000, 400, F32, 128, 0, 0), (6, 200, 16384, F32, 64, 0, 0), (2, 200, 16384, F32, 64, 0, 0), (2, 96, 33000, BF16, 32, 1, 0), (1, 64, 33000, F32, 64, 0, 0), (3, 130, 33000, F16, 128, 1, 1), (16, 200, 17000, F32, 64, 0, 0),
    (20, 300, 500, F32, 32, 1, 0), (40, 300, 500, F32, 32, 0, 1), (32, 9000, 70, F32, 128, 0, 0), (64, 9000, 70, BF16, 128, 1, 0), (48, 300, 20000, F16, 32, 0, 0),
    (1, 4096, 128256, BF16, 32, 0, 0), (6, 4096, 128257, F16, 128, 1, 0), (1, 4090, 128256, F32, 64, 0, 0),
    (64, 771, 129, F32, 128, 1, 0), (65, 260, 50, BF16, 32, 1, 0), (200, 96, 33, F32, 32, 0, 1), (1, 12287, 9, F32, 32, 1, 0), (8, 160, 30000, BF16, 32, 1, 0),
]


def make(case, seed=0):
    m, k, o, dtype, group, bias, relu = case
    g = torch.Generator(device=DEV).manual_seed(seed + m * k + o)
    x = torch.randn((m, k), generator=g, device=DEV).to(dtype)
    codes = torch.randint(256, (o, (k + 1) // 2), generator=g, device=DEV, dtype=torch.uint8)  # with k odd: a last half to ignore
    scales = (torch.rand((o, -(-k // group)), generator=g, device=DEV) + 0.5).div(math.sqrt(8 * k)).to(BF16)
    b = torch.randn(o, generator=g, device=DEV).to(dtype) if bias else None
    return x, codes, scales, b


def run(case, x, codes, scales, b, first=0):
    m, k, o, dtype, group, bias, relu = case
    d = lib.q4_desc_create(lib.Q4Params(m, k, o, dtype, group, bias, relu))
    print(lib.q4_desc_kernel_names(d), flush=True)
    size = lib.q4_desc_packed_bytes(d)
    space = torch.full((size + 64,), 0xEE, device=DEV, dtype=torch.uint8)
    packed = space[:size]
    lib.q4_pack(d, codes, scales, packed)
    assert (space[size:] == 0xEE).all()
    ws_bytes = lib.q4_desc_workspace_bytes(d)
    ws = torch.full((ws_bytes // 4 + 16,), math.nan, device=DEV)
    buffer = torch.full((first + m * o + 8,), math.nan, device=DEV, dtype=dtype)
    y = buffer[first:first + m * o].view(m, o)
    lib.q4_forward(d, x, packed, b, y, ws[:(ws_bytes + 3) // 4])
    assert torch.isnan(ws[(ws_bytes + 3) // 4:]).all()
    assert torch.isnan(buffer[:first]).all() and torch.isnan(buffer[first + m * o:]).all()
    again = torch.empty_like(y)
    lib.q4_forward(d, x, packed, b, again, ws)
    assert torch.equal(again.nan_to_num(7.0), y.nan_to_num(7.0))
    return y


def check(case, x, codes, scales, b, y):
    m, k, o, dtype, group, bias, relu = case
    want = tokens.q4_forward(x, codes, scales, b, k, group, relu)
    size = x.double().abs() @ tokens.q4_weights(codes, scales, k, group).abs().t().contiguous()
    tol = size * (k / 32 + 160) * 2.0 ** -24 + want.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -23)
    tol += (b.double().abs() * 2.0 ** -23 if bias else 0.0) + (2.0 ** -25 if dtype is F16 else 2.0 ** -126)
    off = (y.double() - want).abs()
    assert bool((off <= tol).all()), (float(off.max()), int((off > tol).sum()))


@pytest.mark.parametrize("case", CASES, ids=["%dx%d-%d-%s-g%d-b%d-r%d" % (c[0], c[1], c[2], str(c[3])[6:], *c[4:]) for c in CASES])
def test_parity(case):
    x, codes, scales, b = make(case)
    check(case, x, codes, scales, b, run(case, x, codes, scales, b))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_unaligned_blobs(dtype):
    case = (3, 264, 48, dtype, 32, 1, 0)
    x, codes, scales, b = make(case)
    place = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)
    x, codes, scales, b = place(x), place(codes), place(scales), place(b)
    check(case, x, codes, scales, b, run(case, x, codes, scales, b, first=1))


def test_every_code_and_input_place():
    """One input of one at a time: each output is the weight itself, scale times value, exact in fp32."""
    k, o = 160, 48
    case = (k, k, o, F32, 32, 0, 0)
    _, codes, scales, _ = make(case)
    y = run(case, torch.eye(k, device=DEV), codes, scales, None)
    assert torch.equal(y.double(), tokens.q4_weights(codes, scales, k, 32).t())


def test_fp32_inputs_take_part_with_all_their_bits():
    """Inputs that differ in their last bit only, under weights 1 and -1: the difference comes out exactly."""
    k = 64
    x = torch.full((1, k), 0.0, device=DEV)
    x[0, 0], x[0, 1] = 1.0 + 2.0 ** -23, 1.0
    codes = torch.full((1, k // 2), 0xA2, device=DEV, dtype=torch.uint8)  # 1, -1, 1, -1 ...
    scales = torch.ones((1, 2), device=DEV, dtype=BF16)
    assert float(run((1, k, 1, F32, 32, 0, 0), x, codes, scales, None)) == 2.0 ** -23


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_not_a_number_and_infinity_stay_in_their_rows(dtype):
    case = (20, 200, 40, dtype, 64, 0, 0)
    x, codes, scales, _ = make(case)
    codes |= 0x22  # no zero weights
    x[3, 5], x[7, 150], x[18, 0] = math.nan, math.inf, -math.inf
    x[19] = torch.finfo(dtype).max
    y = run(case, x, codes, scales * 2.0 ** -4, None)
    assert torch.isnan(y[3]).all() and torch.isinf(y[7]).all() and torch.isinf(y[18]).all()
    good = [r for r in range(19) if r not in (3, 7, 18)]
    check((16,) + case[1:], x[good], codes, scales * 2.0 ** -4, None, y[good])


def test_one_packing_serves_other_batches_streams_and_graphs():
    k, o, group = 500, 130, 64
    _, codes, scales, _ = make((1, k, o, BF16, group, 0, 0))
    packed = None
    for m, dtype in ((1, BF16), (7, F16), (64, F32)):
        case = (m, k, o, dtype, group, 0, 0)
        x = make(case, seed=3)[0]
        d = lib.q4_desc_create(lib.Q4Params(m, k, o, dtype, group))
        if packed is None:
            packed = torch.empty(lib.q4_desc_packed_bytes(d), device=DEV, dtype=torch.uint8)
            lib.q4_pack(d, codes, scales, packed)
        ws = torch.empty(lib.q4_desc_workspace_bytes(d) // 4 + 1, device=DEV)
        y = torch.empty((m, o), device=DEV, dtype=dtype)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        lib.q4_forward(d, x, packed, None, y, ws, side)
        side.synchronize()
        check(case, x, codes, scales, None, y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lib.q4_forward(d, x, packed, None, y, ws)
        for k_ in range(3):
            x.normal_()
            graph.replay()
            replayed = y.clone()
            lib.q4_forward(d, x, packed, None, y, ws)
            torch.cuda.synchronize()
            assert torch.equal(replayed, y)
            check(case, x, codes, scales, None, y)


def test_refusals_on_the_device():
    d = lib.q4_desc_create(lib.Q4Params(2, 40, 9, BF16, 32, 1, 0))
    x, codes, scales, b = make((2, 40, 9, BF16, 32, 1, 0))
    packed = torch.empty(lib.q4_desc_packed_bytes(d), device=DEV, dtype=torch.uint8)
    ws = torch.empty(lib.q4_desc_workspace_bytes(d) // 4 + 1, device=DEV)
    y = torch.empty((2, 9), device=DEV, dtype=BF16)
    for wrong, error in ((dict(codes=codes[:, :-1].contiguous()), ValueError), (dict(scales=scales.float()), TypeError),
                         (dict(packed=packed[:-1]), ValueError), (dict(packed=packed.cpu()), TypeError)):
        with pytest.raises(error):
            lib.q4_pack(d, **{**dict(codes=codes, scales=scales, packed=packed), **wrong})
    lib.q4_pack(d, codes, scales, packed)
    shifted = torch.cat([packed.new_zeros(1), packed])[1:]
    for wrong, error in ((dict(x=x.float()), TypeError), (dict(x=x[:1]), ValueError), (dict(bias=None), lib.ConvError),
                         (dict(packed=shifted), lib.ConvError), (dict(y=y.t()), TypeError), (dict(x=x.cpu()), TypeError)):
        with pytest.raises(error):
            lib.q4_forward(d, **{**dict(x=x, packed=packed, bias=b, y=y, ws=ws), **wrong})
    none = lib.q4_desc_create(lib.Q4Params(0, 40, 9, BF16, 32, 0, 0))
    lib.q4_forward(none, x[:0], packed, None, y[:0], ws)


# fp32 rows laid out as operands beforehand in each of the small shapes, for each group; batches of many 64s of rows.
MORE_CASES = [
    (1, 4096, 4096, F32, 64, 0, 0), (3, 1500, 500, F32, 32, 1, 0), (4, 2000, 777, F32, 128, 0, 1), (16, 3001, 600, F32, 32, 0, 0), (5, 1300, 1000, F32, 64, 1, 1),
    (8, 4096, 8000, F32, 64, 1, 0), (5, 130, 9000, F32, 32, 0, 0), (16, 2047, 5001, F32, 128, 0, 1), (7, 1500, 4100, F32, 32, 1, 0),
    (512, 96, 333, F32, 32, 1, 0), (1000, 640, 300, BF16, 128, 1, 1), (130, 300, 3001, F16, 64, 0, 0), (257, 1111, 70, F32, 64, 0, 0), (2049, 130, 40, BF16, 32, 0, 0),
]


@pytest.mark.parametrize("case", MORE_CASES, ids=["%dx%d-%d-%s-g%d-b%d-r%d" % (c[0], c[1], c[2], str(c[3])[6:], *c[4:]) for c in MORE_CASES])
def test_more_shapes(case):
    test_parity(case)


@pytest.mark.parametrize("m", [1, 20])
@pytest.mark.parametrize("dtype,size,scale", [(F32, 2.0 ** -100, 2.0 ** 60), (F32, 2.0 ** -112, 2.0 ** 60), (F32, 2.0 ** -122, 2.0 ** 60),
                                              (F32, 2.0 ** -128, 2.0 ** 70), (F32, 2.0 ** -140, 2.0 ** 80), (BF16, 2.0 ** -124, 2.0 ** 60),
                                              (BF16, 2.0 ** -130, 2.0 ** 70), (F16, 2.0 ** -14, 2.0 ** 8), (F16, 2.0 ** -21, 2.0 ** 12)])
def test_small_and_subnormal_inputs(m, dtype, size, scale):
    """As the others' bound, and what lies below 2^-133 of each fp32 input (2^-133 of it at most) times its weight."""
    case = (m, 1500, 40, dtype, 64, 0, 0)
    x, codes, scales, _ = make(case)
    x, scales = (x.double() * size).to(dtype), (scales.double() * scale).to(BF16)
    y = run(case, x, codes, scales, None)
    want = tokens.q4_forward(x, codes, scales, None, 1500, 64, 0)
    weights = tokens.q4_weights(codes, scales, 1500, 64).abs()
    tol = x.double().abs() @ weights.t().contiguous() * (1500 / 32 + 160) * 2.0 ** -24 + want.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -23)
    tol += (weights.sum(1) * 2.0 ** -133 if dtype is F32 else 0.0) + (2.0 ** -25 if dtype is F16 else 2.0 ** -126)
    if dtype is not F32 or size > 2.0 ** -124:  # (below, what an fp32 input loses is a good part of it, or all)
        assert float(want.abs().max()) > 16 * float(tol.max())
    assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,size,scale", [(F32, 2.0 ** 118, 2.0 ** -16), (BF16, 2.0 ** 118, 2.0 ** -16), (F16, 65504.0, 2.0 ** -12)])
def test_large_inputs(dtype, size, scale, group):
    """The greatest sums that the header promises: every input as large as it may be, weights of 6 and -6 scaled down, one sign and both."""
    case = (3, 512, 40, dtype, group, 0, 0)
    x, codes, scales, _ = make(case)
    x = torch.where(x > 0, size, -size).to(dtype)
    x[0] = size
    codes[:20], codes[20:] = 0x77, 0xF7
    scales = torch.full_like(scales, scale)
    scales[:, 1::2] = -scale / 2
    check(case, x, codes, scales, None, run(case, x, codes, scales, None))


def test_as_many_outputs_as_there_may_be():
    """2^30 - 1 outputs of one input: 2^32 vectors of packed codes (64 GB), more than a launch has threads."""
    o = (1 << 30) - 1
    d = lib.q4_desc_create(lib.Q4Params(1, 1, o, BF16, 128, 0, 0))
    g = torch.Generator(device=DEV).manual_seed(5)
    codes = torch.randint(16, (o, 1), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.ones((o, 1), device=DEV, dtype=BF16)
    packed = torch.empty(lib.q4_desc_packed_bytes(d), device=DEV, dtype=torch.uint8)
    lib.q4_pack(d, codes, scales, packed)
    y = torch.full((1, o), math.nan, device=DEV, dtype=BF16)
    lib.q4_forward(d, torch.full((1, 1), 2.0, device=DEV, dtype=BF16), packed, None, y)
    value = 2 * tokens.q4_values(torch.arange(16, device=DEV, dtype=torch.uint8)[:, None], 1)[:, 0].to(BF16)
    for at in range(0, o, 1 << 26):
        assert torch.equal(y[0, at:at + (1 << 26)], value[codes[at:at + (1 << 26), 0].int()]), at

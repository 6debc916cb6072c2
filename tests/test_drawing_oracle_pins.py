"""The oracle of drawing tokens and of layers in 8 bits against hand-worked values and definitions; and planted mistakes that these checks have to notice."""
import math
import operator

import pytest
import torch

from oracle import tokens


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


ROW = torch.tensor([0.0, math.log(4), math.log(2), -math.inf, math.log(4), 0.0], dtype=torch.float64)  # weights 1/4 1 1/2 0 1 1/4


@pytest.mark.parametrize("limits,kept", [
    (dict(), [1 / 4, 1, 1 / 2, 0, 1, 1 / 4]), (dict(top_k=1), [0, 1, 0, 0, 0, 0]), (dict(top_k=2), [0, 1, 0, 0, 1, 0]), (dict(top_k=4), [1 / 4, 1, 1 / 2, 0, 1, 0]),
    (dict(top_k=6), [1 / 4, 1, 1 / 2, 0, 1, 1 / 4]), (dict(top_k=-1), [1 / 4, 1, 1 / 2, 0, 1, 1 / 4]), (dict(top_p=0.0), [0, 1, 0, 0, 0, 0]),
    (dict(top_p=0.34), [0, 1, 0, 0, 1, 0]), (dict(top_p=0.7), [0, 1, 1 / 2, 0, 1, 0]), (dict(top_p=0.9), [1 / 4, 1, 1 / 2, 0, 1, 0]),
    (dict(top_k=3, top_p=0.7), [0, 1, 0, 0, 1, 0]), (dict(min_p=0.3), [0, 1, 1 / 2, 0, 1, 0]), (dict(min_p=2.0), [0, 1, 0, 0, 1, 0]),
    (dict(min_p=-1.0), [1 / 4, 1, 1 / 2, 0, 1, 1 / 4]), (dict(scale=2.0), [1 / 16, 1, 1 / 4, 0, 1, 1 / 16]), (dict(scale=2.0, top_p=0.9), [0, 1, 1 / 4, 0, 1, 0])])
def test_worked_limits(limits, kept):
    got = tokens.kept_weights(ROW, **limits)
    assert got == pytest.approx(kept, abs=1e-15)


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.08, 0), (0.09, 1), (0.41, 1), (0.42, 2), (0.58, 2), (0.59, 4), (0.91, 4), (0.92, 5), (1.0, 5)])
def test_worked_draws(u, token):
    got, logp = tokens.draw_row(ROW, u)
    assert got == token and logp == pytest.approx(math.log([1 / 4, 1, 1 / 2, 0, 1, 1 / 4][token] / 3), abs=1e-14)


def test_rows_without_a_distribution():
    inf, nan = math.inf, math.nan
    assert tokens.draw_row(torch.full((3,), -inf), 0.5) == (-1, -inf)
    for row, u, more in (([0.0, nan], 0.5, {}), ([inf, 0.0], 0.5, {}), ([0.0], -0.1, {}), ([0.0], 1.1, {}), ([0.0], nan, {}), ([0.0], 0.5, dict(scale=0.0)),
                         ([0.0], 0.5, dict(scale=nan)), ([0.0], 0.5, dict(top_p=nan)), ([0.0], 0.5, dict(min_p=nan)), ([0.0], 0.5, dict(scale=2.0 ** 61))):
        token, logp = tokens.draw_row(torch.tensor(row), u, **more)
        assert token == -1 and math.isnan(logp)


def test_many_rows_as_one_by_one():
    rows, vocab = 300, 23
    x = (rand(rows, vocab) * 2).round(decimals=1)  # with equal ones
    x[::7, ::3] = -math.inf
    g = torch.Generator().manual_seed(1)
    pick = lambda values, t=torch.float32: torch.tensor(values, dtype=t)[torch.randint(len(values), (rows,), generator=g)]
    u, scale, k = torch.rand(rows, generator=g), pick((0.5, 1.0, 2.0)), pick((0, 1, 4, 22, 100, -2), torch.int32)
    p, q = pick((1.0, 0.5, 0.9, 0.0, 3.0)), pick((0.0, 0.05, 0.5, 2.0, -1.0))
    token, logp = tokens.draw(x, u, scale, k, p, q)
    for r in range(rows):
        want = tokens.draw_row(x[r], float(u[r]), float(scale[r]), int(k[r]), float(p[r]), float(q[r]))
        assert int(token[r]) == want[0] and float(logp[r]) == pytest.approx(want[1], abs=1e-12)


def test_planted_mistakes_in_draws_are_noticed():
    """top-p before top-k, and a strict border: the worked limits tell them apart."""
    def top_p_first(w, k, p):
        order = sorted(range(len(w)), key=lambda i: (-w[i], i))
        whole, kept, reached = sum(w), [], 0.0
        for i in order:
            kept.append(i)
            reached += w[i]
            if reached >= p * whole:
                break
        return [w[i] if i in kept[:k] else 0.0 for i in range(len(w))]
    full = tokens.kept_weights(ROW)
    assert top_p_first(full, 3, 0.7) != pytest.approx(tokens.kept_weights(ROW, top_k=3, top_p=0.7))


def limits_by(row, p, q, u, reached, least, passed):
    """Tokens that top-p and min-p keep and the token drawn, with the three borders' comparisons given; equal logits, whose sums are exact."""
    order, kept, w = range(len(row)), [], 0.0
    for _ in order:
        if kept and reached(w, p * len(row)):
            break
        kept.append(len(kept))
        w += 1.0
    kept = [i for i in kept if least(1.0, q)]
    drawn, sums = (kept or [-1])[-1], 0.0
    for i in kept:
        sums += 1.0
        if passed(sums, u * len(kept)):
            drawn = i
            break
    return kept, drawn


@pytest.mark.parametrize("which", [None, "top_p", "min_p", "u"])
def test_planted_strict_borders_are_noticed(which):
    """Eight equal logits under borders that their sums meet exactly: top-p is reached by as much as it asks for, min-p keeps what is equal, u is to be passed."""
    row = torch.zeros(8, dtype=torch.float64)
    got = limits_by(row, 0.5, 1.0, 0.5, operator.gt if which == "top_p" else operator.ge, operator.gt if which == "min_p" else operator.ge,
                    operator.ge if which == "u" else operator.gt)
    w = tokens.kept_weights(row, top_p=0.5, min_p=1.0)
    want = [i for i, v in enumerate(w) if v > 0], tokens.draw_row(row, 0.5, top_p=0.5, min_p=1.0)[0]
    assert want == ([0, 1, 2, 3], 2)
    assert (got == want) == (which is None)
    full = lambda v, t=torch.float32: torch.full((1,), v, dtype=t)
    token, logp = tokens.draw(row[None], full(0.5), full(1.0), full(0, torch.int32), full(0.5), full(1.0))
    assert (int(token), float(logp)) == (2, pytest.approx(math.log(1 / 4)))


def eight_bits_by(x, scale_of, nearest):
    scale = torch.tensor([scale_of(float(v)) for v in x.abs().amax(1)], dtype=torch.float64)
    return nearest(x.double() / scale[:, None]), scale


@pytest.mark.parametrize("which", [None, "scale of 24 bits", "scale rounded to nearest", "halves up", "halves away from 0"])
def test_planted_mistakes_in_eight_bits_are_noticed(which):
    def up(most):
        fraction, exponent = math.frexp(most / 127)
        return math.ldexp(math.ceil(fraction * 256), exponent - 8)

    def near(most):
        fraction, exponent = math.frexp(most / 127)
        return math.ldexp(round(fraction * 256), exponent - 8)
    scale_of = {"scale of 24 bits": lambda most: most / 127, "scale rounded to nearest": near}.get(which, up)
    nearest = {"halves up": lambda t: torch.floor(t + 0.5), "halves away from 0": lambda t: torch.sign(t) * torch.floor(t.abs() + 0.5)}.get(which, torch.round)
    x = torch.tensor([[127.0, 0.5, 1.5, -2.5, -3.5], [254.0, 1.0, -3.0, 3.1, 0.0], [128.25, 1.0, 64.0, -7.0, 0.0]])
    codes, scale = tokens.eight_bits(x)
    got_codes, got_scale = eight_bits_by(x, scale_of, nearest)
    assert (torch.equal(got_codes, codes) and torch.equal(got_scale, scale)) == (which is None)


@pytest.mark.parametrize("which", [None, "scale of the row left out", "scale of the output left out", "scale taken twice", "bias gradient with the scale"])
def test_planted_mistakes_in_gradients_of_eight_bits_are_noticed(which):
    x, w, dz = rand(5, 12), rand(7, 12, seed=1), rand(5, 7, seed=2)
    (c, s), (v, t) = tokens.eight_bits(x), tokens.eight_bits(w)
    wanted = tokens.i8_backward_filter(c, s, dz) + (tokens.i8_backward_data(v, t, dz),)
    row = {"scale of the row left out": torch.ones_like(s), "scale taken twice": s * s}.get(which, s)
    out = torch.ones_like(t) if which == "scale of the output left out" else t
    got = (dz * row[:, None]).t() @ c, (dz * s[:, None] if which == "bias gradient with the scale" else dz).sum(0), (dz * out[None]) @ v
    assert all(torch.allclose(a, b, rtol=1e-12) for a, b in zip(got, wanted)) == (which is None)


def test_worked_rows_in_eight_bits():
    x = torch.tensor([[127.0, 0.5, 1.5, -2.5, 126.5], [254.0, 1.0, -3.0, 3.1, 0.0], [0.0] * 5, [128.0, 0, 0, 0, 0], [1.0, -math.inf, 0, 0, 0]])
    codes, scale = tokens.eight_bits(x)
    assert codes[0].tolist() == [127, 0, 2, -2, 126] and float(scale[0]) == 1.0
    assert codes[1].tolist() == [127, 0, -2, 2, 0] and float(scale[1]) == 2.0
    assert codes[2].tolist() == [0] * 5 and float(scale[2]) == 2.0 ** -126
    assert float(scale[3]) == 130 / 128 and codes[3, 0] == 126  # 128 / 127 = 1.00787 is above 129 / 128 = 1.00781
    assert math.isnan(float(scale[4])) and codes[4].tolist() == [0] * 5


@pytest.mark.parametrize("seed", range(4))
def test_eight_bits_is_the_nearest_and_its_scale_the_smallest(seed):
    x = (rand(40, 17, seed=seed) * torch.exp(rand(40, 1, seed=seed + 9) * 10)).float()
    codes, scale = tokens.eight_bits(x)
    most = x.double().abs().amax(1)
    assert bool((127 * scale >= most).all()) and bool((codes.abs() <= 127).all())
    fraction, exponent = torch.frexp(scale)
    assert bool((fraction * 256 == (fraction * 256).round()).all())
    smaller = torch.ldexp(torch.where(fraction == 0.5, fraction * 256 - 0.5, fraction * 256 - 1), exponent - 8)
    assert bool((127 * smaller < most).all())
    assert bool(((codes * scale[:, None] - x.double()).abs() <= scale[:, None] / 2).all())


def test_layer_and_gradients_are_those_of_the_values():
    x, w, dz = rand(5, 12), rand(7, 12, seed=1), rand(5, 7, seed=2)
    bias = rand(7, seed=3)
    (c, s), (v, t) = tokens.eight_bits(x), tokens.eight_bits(w)
    xq, wq = (c * s[:, None]).requires_grad_(), (v * t[:, None]).requires_grad_()
    b = bias.clone().requires_grad_()
    y = xq @ wq.t() + b
    assert torch.allclose(tokens.i8_forward(c, s, v, t, bias, 0), y.detach(), rtol=1e-13)
    assert torch.equal(tokens.i8_forward(c, s, v, t, bias, 1) > 0, y.detach() > 0)
    y.backward(dz)
    dw, db = tokens.i8_backward_filter(c, s, dz)
    assert torch.allclose(dw, wq.grad, rtol=1e-12) and torch.allclose(db, b.grad, rtol=1e-12)
    assert torch.allclose(tokens.i8_backward_data(v, t, dz), xq.grad, rtol=1e-12)

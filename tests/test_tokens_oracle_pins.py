"""The oracle of the token policy's operators against hand-worked values, closed forms, differences and the framework's other
oracle; and planted mistakes that these checks have to notice."""
import math

import numpy as np
import pytest
import torch

from oracle import policy_gradient as pgo
from oracle import tokens


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_worked_row():
    x = torch.tensor([[0.0, math.log(2), math.log(5)]], dtype=torch.float64)
    logp, h = tokens.log_probs(x)
    p = [1 / 8, 2 / 8, 5 / 8]
    assert torch.allclose(logp.exp()[0], torch.tensor(p, dtype=torch.float64), rtol=1e-14)
    assert abs(float(h[0]) + sum(q * math.log(q) for q in p)) < 1e-14
    g = tokens.d_logits(x, torch.tensor([1]), torch.tensor([2.0]), None)
    assert torch.allclose(g[0], torch.tensor([-2 / 8, 2 - 4 / 8, -10 / 8], dtype=torch.float64), rtol=1e-14)
    assert tokens.token_logp(logp, torch.tensor([-1])).item() == 0.0 and tokens.token_logp(logp, torch.tensor([3])).item() == 0.0
    assert tokens.token_logp(logp, torch.tensor([0])).item() == pytest.approx(math.log(1 / 8), abs=1e-14)


def test_uniform_empty_and_masked_rows():
    inf = math.inf
    x = torch.tensor([[3.0] * 4, [-inf] * 4, [-inf, 1.0, -inf, 1.0]])
    logp, h = tokens.log_probs(x, 0.5)
    assert torch.allclose(h, torch.tensor([math.log(4), 0.0, math.log(2)], dtype=torch.float64), atol=1e-15)
    assert (logp[1] == -inf).all() and logp[2].tolist()[::2] == [-inf, -inf]
    g = tokens.d_logits(x, torch.tensor([0, 1, 0]), torch.ones(3), torch.ones(3), 0.5)
    assert torch.isfinite(g).all() and g[1].tolist() == [0, 0.5, 0, 0] and g[2].tolist()[0] == 0.5 and g[2, 2] == 0
    lowest = torch.full((1, 5), torch.finfo(torch.float32).min)
    assert torch.allclose(tokens.log_probs(lowest, 1.5)[0].exp(), torch.full((1, 5), 0.2, dtype=torch.float64))


def test_order_of_alternatives():
    x = torch.tensor([[1.0, -0.0, 7.0, 0.0, 7.0, -math.inf, math.nan]])
    assert tokens.top_tokens(x, 7)[0].tolist() == [6, 2, 4, 0, 1, 3, 5]
    assert tokens.top_tokens(torch.where(torch.isnan(x), -x, x), 7)[0].tolist() == [6, 2, 4, 0, 1, 3, 5]


def loss(x, token, d_logp, d_entropy, scale):
    logp, h = tokens.log_probs(x, scale)
    return (tokens.token_logp(logp, token) * d_logp).sum() + (h * d_entropy).sum()


def check_gradient(gradient):
    x, token = rand(3, 6), torch.tensor([2, -1, 5])
    d_logp, d_entropy, scale = rand(3, seed=1), rand(3, seed=2), 0.75
    x[0, 4] = -math.inf
    g = gradient(x, token, d_logp, d_entropy, scale)
    for r in range(3):
        for i in range(6):
            if not math.isfinite(float(x[r, i])):
                assert float(g[r, i]) == 0.0
                continue
            hi, lo = x.clone(), x.clone()
            hi[r, i] += 1e-6
            lo[r, i] -= 1e-6
            diff = float(loss(hi, token, d_logp, d_entropy, scale) - loss(lo, token, d_logp, d_entropy, scale)) / 2e-6
            assert abs(diff - float(g[r, i])) < 1e-8


def test_gradient_is_that_of_the_loss():
    check_gradient(tokens.d_logits)


@pytest.mark.parametrize("mutant", ["scale", "entropy", "sign", "token"])
def test_planted_mistakes_in_the_gradient_are_noticed(mutant):
    def wrong(x, token, d_logp, d_entropy, scale):
        if mutant == "scale":
            return tokens.d_logits(x, token, d_logp, d_entropy, scale) / scale
        if mutant == "entropy":
            return tokens.d_logits(x, token, d_logp, None, scale)
        if mutant == "sign":
            return tokens.d_logits(x, token, d_logp, -d_entropy, scale)
        return tokens.d_logits(x, token.clamp(min=0), d_logp, d_entropy, scale)
    with pytest.raises(AssertionError):
        check_gradient(wrong)


def test_gradient_agrees_with_the_policy_gradient_oracle():
    """bottom_diff of the Softmax model is -R times the derivative of the action's log probability."""
    x, action, reward = rand(5, 4), torch.tensor([0, 3, 1, 2, 2]), rand(5, seed=3)
    _, dlogps = pgo.softmax_dlogps(x.numpy(), action.numpy())
    want = pgo.bottom_diff(dlogps, reward.numpy(), False)
    got = tokens.d_logits(x, action, -reward, None)
    assert np.allclose(got.numpy(), want, atol=1e-13)


def test_clip():
    grads = [torch.tensor([3.0, 0.0]), torch.zeros(0), torch.tensor([[4.0]], dtype=torch.bfloat16)]
    norm, out = tokens.clip(grads, 10.0)
    assert norm == 5.0 and out[0].tolist() == [3.0, 0.0]
    norm, out = tokens.clip(grads, 1.0)
    assert out[0].tolist() == pytest.approx([0.6, 0.0]) and out[2].item() == pytest.approx(0.8)
    assert math.sqrt(sum(float(t.square().sum()) for t in out)) == pytest.approx(1.0)


def test_q4_values_are_the_sixteen():
    codes = torch.tensor([[0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]], dtype=torch.uint8)
    want = [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]
    assert tokens.q4_values(codes, 16)[0].tolist() == want
    assert tokens.q4_values(codes, 3)[0].tolist() == want[:3]


def test_q4_forward_by_hand():
    codes = torch.tensor([[0x42, 0x03], [0xF1, 0x0A]], dtype=torch.uint8)  # 1 2 1.5 | 0.5 -6 -1
    scales = torch.tensor([[2.0], [0.5]], dtype=torch.bfloat16)
    x = torch.tensor([[1.0, 2.0, 3.0]])
    y = tokens.q4_forward(x, codes, scales, torch.tensor([1.0, 1.0]), 3, 32, 0)
    assert y.tolist() == [[2 * (1 + 4 + 4.5) + 1, 0.5 * (0.5 - 12 - 3) + 1]]
    assert tokens.q4_forward(x, codes, scales, None, 3, 32, 1)[0, 1] == 0
    # a second group takes its own scale
    codes = torch.full((1, 17), 0x22, dtype=torch.uint8)
    scales = torch.tensor([[1.0, 8.0]], dtype=torch.bfloat16)
    assert tokens.q4_forward(torch.ones(1, 34), codes, scales, None, 34, 32, 0).item() == 32 + 2 * 8

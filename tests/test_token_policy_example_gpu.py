"""The example that runs the token policy's operators together: its gradients against the formulas in 64 bits, and that it learns."""
import os
import sys

import pytest
import torch

from oracle import tokens

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import token_policy  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("k,group", [(64, 32), (65, 32), (97, 64), (5, 128)])
def test_quantised_weights_are_the_nearest(k, group):
    w = torch.randn(7, k, generator=torch.Generator().manual_seed(k))
    codes, scales = token_policy.quantise(w, group)
    assert codes.shape == (7, (k + 1) // 2) and scales.shape == (7, -(-k // group))
    got = tokens.q4_weights(codes, scales, k, group)
    step = scales.double()[:, torch.arange(k) // group]
    assert float(((got - w.double()).abs() / step).max()) <= 1.0 + 2.0 ** -7 * 6  # half of the widest gap, 4 to 6, and the scale's rounding


@pytest.mark.gpu
def test_gradients_against_the_formulas():
    """fp32 throughout: a logit is off by at most 96 2^-23 of its terms' size (below 2^-12 here), a gradient entry by the sum over rows
    of that in each term: 2^-9 of the largest entry covers them."""
    torch.manual_seed(3)
    rows, features, vocab = 40, 96, 333
    p = token_policy.Policy(rows, features, vocab, limit=1e9, device=DEV)
    x = torch.randn(rows, features, device=DEV)
    discounted = torch.randn(rows, device=DEV)
    token = p.play(x, torch.rand((rows, vocab), device=DEV).clamp(min=1e-20))
    codes, scales = token_policy.quantise(p.w, 32)
    played = tokens.q4_forward(x, codes, scales, p.b, features, 32, 0)
    assert float((p.logits.double() - played).abs().max()) < 2.0 ** -12
    logp, _ = tokens.log_probs(p.logits)
    assert float((p.logp.double() - tokens.token_logp(logp, token)).abs().max()) < 1e-4
    p.gradients(x, token, discounted)
    logits = x.double() @ p.w.double().t().contiguous() + p.b.double()
    d = tokens.d_logits(logits, token, -discounted / rows, torch.full_like(discounted, -p.bonus / rows))
    for got, want in zip(p.grads, (d.t().contiguous() @ x.double(), d.sum(0))):
        assert float((got.double() - want).abs().max()) < 2.0 ** -9 * float(want.abs().max())
    norm = float(p.norm)
    assert abs(norm - tokens.clip(p.grads, 1e9)[0]) < 1e-5 * norm
    p.limit = norm / 3
    p.gradients(x, token, discounted)
    assert abs(tokens.clip(p.grads, 1e9)[0] - norm / 3) < 1e-5 * norm


@pytest.mark.gpu
def test_it_learns():
    rewards = token_policy.train(rounds=40, say=None, device=DEV)
    assert sum(rewards[-5:]) / 5 > 0.5 > 0.1 > rewards[0]

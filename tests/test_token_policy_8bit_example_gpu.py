"""The example that plays and trains a policy in 8 bits: its draws and gradients against the formulas in 64 bits, and that it runs."""
import math
import os
import sys

import pytest
import torch

from oracle import tokens

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import token_policy_8bit  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_draws_and_gradients_against_the_formulas():
    """Each call against the oracle on that call's own inputs.  fp32 throughout: a sum of n terms is within (n / 32 * 3 + 40) 2^-24 of its terms'
    magnitudes; 2^-15 covers 512 rows, 333 and 150 inputs (96 2^-24 at most)."""
    torch.manual_seed(3)
    rows, features, hidden, vocab = 96, 40, 150, 333
    p = token_policy_8bit.Policy(rows, features, hidden, vocab, limit=1e9, device=DEV)
    x, u, discounted = torch.randn(rows, features, device=DEV), torch.rand(rows, device=DEV), torch.randn(rows, device=DEV)
    token = p.play(x, u)
    close = lambda got, want, size: bool(((got.double() - want).abs() <= 2.0 ** -15 * size + 1e-30).all())
    for layer, at, relu in ((p.first, x, 1), (p.second, p.first.y, 0)):
        k = at.shape[1]
        codes, scale = tokens.eight_bits(at)
        assert torch.equal(layer.codes[:, :k].double(), codes) and torch.equal(layer.scale.double(), scale)
        codes_w, scale_w = tokens.eight_bits(layer.w)
        assert torch.equal(layer.w_codes[:, :k].double(), codes_w)
        size = tokens.i8_forward(codes.abs(), scale, codes_w.abs(), scale_w, layer.b.abs(), 0)
        assert close(layer.y, tokens.i8_forward(codes, scale, codes_w, scale_w, layer.b, relu), size)
    logits = p.second.y.clone()
    want, want_logp = tokens.draw(logits, u, torch.ones(rows, device=DEV), p.top_k, p.top_p, torch.zeros(rows, device=DEV))
    assert torch.equal(token, want) and bool(((p.drawn.double() - want_logp).abs() <= 2.0 ** -22 * (1 + want_logp.abs())).all())

    p.gradients(token, discounted)
    dz = tokens.d_logits(logits, token, -discounted / rows, torch.full_like(discounted, -p.bonus / rows))
    assert float((p.d_logits.double() - dz).abs().max()) <= 2.0 ** -20 * float(dz.abs().max())
    gated = torch.where(p.first.y > 0, p.d_hidden, torch.zeros_like(p.d_hidden))
    assert torch.equal(gated, p.d_hidden)
    back = tokens.i8_backward_data(p.second.w_codes[:, :hidden], p.second.w_scale, p.d_logits)
    back_size = tokens.i8_backward_data(p.second.w_codes[:, :hidden].abs(), p.second.w_scale, p.d_logits.abs())
    assert close(p.d_hidden, torch.where(p.first.y > 0, back, torch.zeros_like(back)), back_size)
    for layer, grad in ((p.second, p.d_logits), (p.first, p.d_hidden)):
        k = layer.w.shape[1]
        dw, db = tokens.i8_backward_filter(layer.codes[:, :k], layer.scale, grad)
        size, size_b = tokens.i8_backward_filter(layer.codes[:, :k].abs(), layer.scale, grad.abs())
        assert close(layer.dw, dw, size) and close(layer.db, db, size_b)
    norm = float(p.norm)
    assert abs(norm - tokens.clip(p.grads, 1e9)[0]) < 1e-5 * norm
    p.limit = norm / 3
    p.gradients(token, discounted)
    assert abs(tokens.clip(p.grads, 1e9)[0] - norm / 3) < 1e-5 * norm


def test_a_step_lowers_the_loss_as_its_gradient_says():
    """Along the gradient of the output layer's bias, which 8 bits leave as it is: the loss's difference over the step against the gradient."""
    torch.manual_seed(5)
    rows, features, hidden, vocab = 64, 30, 70, 100
    p = token_policy_8bit.Policy(rows, features, hidden, vocab, bonus=0.0, limit=1e9, device=DEV)
    x, u, discounted = torch.randn(rows, features, device=DEV), torch.rand(rows, device=DEV), torch.randn(rows, device=DEV)
    token = p.play(x, u).clone()
    p.gradients(token, discounted)
    logits, db = p.second.y.double(), p.second.db.double()
    loss = lambda shift: float(-(discounted.double() / rows * tokens.token_logp(tokens.log_probs(logits + shift)[0], token)).sum())
    h = 1e-4
    slope = (loss(h * db) - loss(-h * db)) / (2 * h)
    assert abs(slope - float(db @ db)) <= 1e-4 * float(db @ db)


def test_it_runs():
    rewards = token_policy_8bit.train(rounds=3, say=None, device=DEV)
    assert len(rewards) == 3 and all(math.isfinite(r) for r in rewards)

"""A policy over tokens with a hidden layer, played and trained in 8-bit integers: drawing tokens, the layers and their gradients run
together as a program uses them.

Each round a batch of episodes is played: features go through two InnerProduct layers in 8 bits (``i8_forward``), the first with a ReLU, and the
next token is drawn from the logits with top-k and top-p (``sm_sample``).  A token that its position asks for earns a reward.  Training takes
the loss's gradient by the logits (``lp_forward_backward``) back through the layers: the weights' gradients from the activations that playing
left in 8 bits (``i8_backward_filter``), the hidden activations' from the weights in 8 bits (``i8_backward_data``, ``ip_relu_backward``),
clipping by their global norm (``gn_clip``), and a step; the new weights are rounded to 8 bits (``i8_pack``) for the next round.

    python examples/token_policy_8bit.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1810_02272_amd as lib  # noqa: E402


class Layer:
    """An InnerProduct layer of fp32 weights that is used in 8 bits."""

    def __init__(self, rows, k, o, relu, device):
        f = lambda *shape, dtype=torch.float32: torch.empty(shape, device=device, dtype=dtype)
        self.d = lib.i8_desc_create(lib.I8Params(rows, k, o, torch.float32, 1, relu))
        row = lib.i8_desc_row_bytes(self.d)
        self.w, self.b = torch.randn(o, k, device=device) * k ** -0.5, torch.zeros(o, device=device)
        self.w_codes, self.w_scale = f(o, row, dtype=torch.int8), f(o)
        self.codes, self.scale = f(rows, row, dtype=torch.int8), f(rows)  # what is kept of x
        self.y, self.dw, self.db = f(rows, o), f(o, k), f(o)
        self.pack()

    def pack(self):
        lib.i8_pack(self.d, self.w, self.w_codes, self.w_scale)

    def forward(self, x, ws):
        lib.i8_forward(self.d, x, self.w_codes, self.w_scale, self.b, self.y, self.codes, self.scale, ws)
        return self.y

    def gradients(self, dz, ws):
        lib.i8_backward_filter(self.d, self.codes, self.scale, dz, self.dw, self.db, 0.0, ws)


class Policy:
    def __init__(self, rows, features, hidden, vocab, top_k=20, top_p=0.95, bonus=0.01, limit=1.0, rate=4.0, device="cuda"):
        f = lambda *shape, dtype=torch.float32: torch.empty(shape, device=device, dtype=dtype)
        self.rows, self.bonus, self.limit, self.rate = rows, bonus, limit, rate
        self.first, self.second = Layer(rows, features, hidden, 1, device), Layer(rows, hidden, vocab, 0, device)
        self.gate = lib.ip_desc_create(lib.IpParams(rows, features, hidden, 1, 1))
        self.sm = lib.sm_desc_create(lib.SmParams(rows, vocab))
        self.lp = lib.lp_desc_create(lib.LpParams(rows, vocab))
        self.grads = [self.first.dw, self.first.db, self.second.dw, self.second.db]
        self.gn = lib.gn_desc_create(lib.GnParams([t.numel() for t in self.grads], [t.dtype for t in self.grads]))
        need = [lib.i8_desc_workspace_bytes(self.first.d), lib.i8_desc_workspace_bytes(self.second.d), lib.sm_desc_workspace_bytes(self.sm),
                lib.lp_desc_workspace_bytes(self.lp), lib.gn_desc_workspace_bytes(self.gn)]
        self.ws = f(max(need) // 4 + 1)  # every call's: they follow each other on one stream
        self.top_k, self.top_p = torch.full((rows,), top_k, device=device, dtype=torch.int32), torch.full((rows,), top_p, device=device)
        self.token, self.drawn = f(rows, dtype=torch.int32), f(rows)  # and the log probability that it was drawn with
        self.logp, self.entropy, self.norm = f(rows), f(rows), f(1)
        self.d_logits, self.d_hidden = f(rows, vocab), f(rows, hidden)

    def play(self, x, u):
        """Tokens drawn with the uniform numbers given; leaves the layers' activations in 8 bits."""
        logits = self.second.forward(self.first.forward(x, self.ws), self.ws)
        lib.sm_sample(self.sm, logits, u, None, self.top_k, self.top_p, None, self.token, self.drawn, self.ws)
        return self.token

    def gradients(self, token, discounted):
        """Of the loss on what has just been played, into self.grads, clipped."""
        d_logp, d_entropy = -discounted / self.rows, torch.full_like(discounted, -self.bonus / self.rows)
        lib.lp_forward_backward(self.lp, self.second.y, token, d_logp, d_entropy, self.logp, self.entropy, self.d_logits, self.ws)
        self.second.gradients(self.d_logits, self.ws)
        lib.i8_backward_data(self.second.d, self.second.w_codes, self.second.w_scale, self.d_logits, self.d_hidden, self.ws)
        lib.ip_relu_backward(self.gate, self.first.y, self.d_hidden, self.d_hidden)
        self.first.gradients(self.d_hidden, self.ws)
        lib.gn_clip(self.gn, self.grads, self.limit, None, self.norm, self.ws)

    def step(self):
        for layer in (self.first, self.second):
            layer.w -= self.rate * layer.dw
            layer.b -= self.rate * layer.db
            layer.pack()


def train(episodes=64, steps=8, features=40, hidden=150, vocab=333, rounds=40, gamma=0.5, seed=0, device="cuda", say=print):
    """Position t of an episode asks for token want[t]; returns each round's mean reward."""
    torch.manual_seed(seed)
    rows = episodes * steps
    policy = Policy(rows, features, hidden, vocab, device=device)
    place = torch.arange(steps, device=device).repeat(episodes)
    x = torch.randn(steps, features, device=device)[place]
    want = torch.randint(vocab, (steps,), device=device)[place]
    offsets = torch.arange(0, rows + 1, steps, device=device, dtype=torch.int32)
    discounted = torch.empty(rows, device=device)
    rewards = []
    for r in range(rounds):
        token = policy.play(x, torch.rand(rows, device=device))
        near = 0.1 * ((token - want).abs() <= 8).float()
        reward = (token == want).float() + near - 0.02
        lib.pg_discount_rewards(reward, offsets, gamma, discounted)
        policy.gradients(token, discounted)
        policy.step()
        rewards.append(float(reward.mean()))
        if say and r % 5 == 0:
            say(f"round {r:3d}: mean reward {rewards[-1]:.3f}, log p {float(policy.drawn.mean()):.2f}, "
                f"entropy {float(policy.entropy.mean()):.2f}, gradient norm {float(policy.norm):.3f}")
    return rewards


if __name__ == "__main__":
    train()

"""A policy whose actions are tokens, trained by policy gradient: the operators for it run together as a program uses them.

Each round a batch of episodes is played: the next token's logits come from 4-bit weights (``q4_forward``), the token is drawn
from them, and its log probability and alternatives are kept (``lp_forward``).  A token that its position asks for earns a
reward, discounted over the episode (``pg_discount_rewards``).  Training then goes through the fp32 weights: logits
(``ip_forward``), the gradient of the loss ``-sum R log p - bonus sum H`` (``lp_forward_backward``), the weights' gradients
(``ip_backward_filter``, ``ip_backward_bias``), clipping by their global norm (``gn_clip``), and a step; the new weights are
rounded to 4 bits and packed (``q4_pack``) for the next round.

    python examples/token_policy.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1810_02272_amd as lib  # noqa: E402

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # of the 4-bit type, without its sign


def quantise(w, group):
    """w [o][k] -> codes two a byte, a bf16 scale for each group: each weight to the nearest multiple of its group's scale."""
    o, k = w.shape
    padded = torch.nn.functional.pad(w, (0, -k % group)).view(o, -1, group)
    scales = (padded.abs().amax(2) / VALUES[-1]).clamp(min=1e-20).to(torch.bfloat16)
    ratio = padded / scales.float()[:, :, None]
    values = torch.tensor(VALUES, device=w.device)
    nearest = torch.bucketize(ratio.abs(), (values[1:] + values[:-1]) / 2)
    codes = (nearest + torch.where(ratio < 0, 8, 0)).to(torch.uint8).view(o, -1)[:, :k + k % 2]
    if k % 2:
        codes = torch.nn.functional.pad(codes[:, :k], (0, 1))
    return (codes[:, 0::2] | codes[:, 1::2] << 4).contiguous(), scales


class Policy:
    """An InnerProduct layer from features to the logits of a vocabulary, in fp32 for training and in 4 bits for playing."""

    def __init__(self, rows, features, vocab, top=4, group=32, bonus=0.01, limit=1.0, rate=4.0, device="cuda"):
        f = lambda *shape: torch.empty(shape, device=device)
        self.rows, self.group, self.bonus, self.limit, self.rate = rows, group, bonus, limit, rate
        self.w, self.b = torch.randn(vocab, features, device=device) * 0.02, torch.zeros(vocab, device=device)
        # plans and memory, once
        self.ip = lib.ip_desc_create(lib.IpParams(rows, features, vocab, 1, 0))
        self.q4 = lib.q4_desc_create(lib.Q4Params(rows, features, vocab, torch.float32, group, 1, 0))
        self.play_lp = lib.lp_desc_create(lib.LpParams(rows, vocab, torch.float32, top, 1))
        self.train_lp = lib.lp_desc_create(lib.LpParams(rows, vocab, torch.float32, 0, 1))
        self.grads = [torch.empty_like(self.w), torch.empty_like(self.b)]
        self.gn = lib.gn_desc_create(lib.GnParams([t.numel() for t in self.grads], [t.dtype for t in self.grads]))
        need = [lib.ip_desc_workspace_bytes(self.ip), lib.q4_desc_workspace_bytes(self.q4), lib.lp_desc_workspace_bytes(self.play_lp),
                lib.lp_desc_workspace_bytes(self.train_lp), lib.gn_desc_workspace_bytes(self.gn)]
        self.ws = f(max(need) // 4 + 1)  # every call's: they follow each other on one stream
        self.packed = torch.empty(lib.q4_desc_packed_bytes(self.q4), device=device, dtype=torch.uint8)
        self.logits, self.logp, self.entropy, self.norm = f(rows, vocab), f(rows), f(rows), f(1)
        self.top_logp, self.top_token = f(rows, top), torch.empty((rows, top), device=device, dtype=torch.int32)
        self.pack()

    def pack(self):
        lib.q4_pack(self.q4, *quantise(self.w, self.group), self.packed)

    def play(self, x, noise):
        """Tokens drawn with the noise given (uniform in (0, 1)), scored."""
        lib.q4_forward(self.q4, x, self.packed, self.b, self.logits, self.ws)
        token = (self.logits - torch.log(-torch.log(noise))).argmax(1).int()
        lib.lp_forward(self.play_lp, self.logits, token, self.logp, self.entropy, None, self.top_logp, self.top_token, self.ws)
        return token

    def gradients(self, x, token, discounted):
        """Of the loss, into self.grads, clipped; leaves the tokens' log probabilities under the weights as they are."""
        lib.ip_forward(self.ip, x, self.w, self.b, self.logits, self.ws)
        d_logp, d_entropy = -discounted / self.rows, torch.full_like(discounted, -self.bonus / self.rows)
        lib.lp_forward_backward(self.train_lp, self.logits, token, d_logp, d_entropy, self.logp, self.entropy, self.logits, self.ws)
        lib.ip_backward_filter(self.ip, x, self.logits, self.grads[0], 0.0, self.ws)
        lib.ip_backward_bias(self.ip, self.logits, self.grads[1], 0.0, self.ws)
        lib.gn_clip(self.gn, self.grads, self.limit, None, self.norm, self.ws)

    def step(self):
        self.w -= self.rate * self.grads[0]
        self.b -= self.rate * self.grads[1]
        self.pack()


def train(episodes=64, steps=8, features=96, vocab=333, rounds=40, gamma=0.5, seed=0, device="cuda", say=print):
    """Position t of an episode asks for token want[t]; returns each round's mean reward."""
    torch.manual_seed(seed)
    rows = episodes * steps
    policy = Policy(rows, features, vocab, device=device)
    place = torch.arange(steps, device=device).repeat(episodes)
    x = torch.randn(steps, features, device=device)[place]
    want = torch.randint(vocab, (steps,), device=device)[place]
    offsets = torch.arange(0, rows + 1, steps, device=device, dtype=torch.int32)
    discounted = torch.empty(rows, device=device)
    rewards = []
    for r in range(rounds):
        noise = torch.rand((rows, vocab), device=device).clamp(min=1e-20)
        token = policy.play(x, noise)
        hit = ((policy.top_token == want[:, None]).any(1)).float()  # the token asked for is among the alternatives
        reward = (token == want).float() + 0.1 * hit - 0.02
        lib.pg_discount_rewards(reward, offsets, gamma, discounted)
        policy.gradients(x, token, discounted)
        policy.step()
        rewards.append(float(reward.mean()))
        if say and r % 5 == 0:
            say(f"round {r:3d}: mean reward {rewards[-1]:.3f}, log p {float(policy.logp.mean()):.2f}, "
                f"entropy {float(policy.entropy.mean()):.2f}, gradient norm {float(policy.norm):.3f}")
    return rewards


if __name__ == "__main__":
    train()

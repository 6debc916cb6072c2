"""Oracle for the operators of a policy over tokens (include/mi355lp.h, mi355gn.h, mi355q4.h) -- TEST INFRASTRUCTURE ONLY: torch
in double precision on whatever device the inputs are, written from the definitions.  Nothing in the GPU package may import this module."""
from __future__ import annotations

import math

import torch


def log_probs(logits, scale=1.0):
    """(log p [rows][vocab], entropy [rows]); a row of nothing but -inf has log p = -inf throughout and entropy 0."""
    x = logits.double()
    top = x.amax(1, keepdim=True)
    empty = top == -math.inf
    z = torch.where(empty, torch.full_like(x, -math.inf), (x - top) * scale)  # -inf - -inf is the empty rows' alone
    e = torch.exp(z)
    logp = torch.where(empty, z, z - torch.log(e.sum(1, keepdim=True)))
    p = torch.exp(logp)
    entropy = -torch.where(p == 0, torch.zeros_like(p), p * logp).sum(1)
    return logp, entropy


def token_logp(logp, token):
    """0 where the token counts for nothing."""
    valid = (token >= 0) & (token < logp.shape[1])
    at = torch.where(valid, token, 0).long()[:, None]
    return torch.where(valid, logp.gather(1, at)[:, 0], 0.0)


def top_tokens(logits, top):
    """Indices of the largest logits: NaN first, equal ones by their index."""
    x = torch.where(torch.isnan(logits), torch.full_like(logits, math.nan), logits + 0.0)  # a sort may order by signs of NaN and 0
    return torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]


def d_logits(logits, token, d_logp, d_entropy, scale=1.0):
    logp, entropy = log_probs(logits, scale)
    p = torch.exp(logp)
    valid = (token >= 0) & (token < logits.shape[1])
    w = torch.where(valid, d_logp.double(), 0.0)
    onehot = torch.zeros_like(p).scatter_(1, torch.where(valid, token, 0).long()[:, None], valid.double()[:, None])
    g = w[:, None] * (onehot - p)
    if d_entropy is not None:
        inner = torch.where(p == 0, torch.zeros_like(p), p * (logp + entropy[:, None]))
        g = g - d_entropy.double()[:, None] * inner
    return g * scale


def clip(grads, limit):
    """(norm, outputs in double)."""
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    factor = limit / norm if norm > limit else 1.0
    return norm, [g.double() * factor for g in grads]


def q4_values(codes, k):
    """[num_output][k] from bytes: one sign bit, two exponent bits (bias 1), one mantissa bit; exponent 0 without the leading one."""
    c = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)[:, :k].int()
    sign, exponent, mantissa = c >> 3, (c >> 1) & 3, c & 1
    value = torch.where(exponent == 0, 0.5 * mantissa, torch.ldexp(1.0 + 0.5 * mantissa.double(), exponent - 1).double())
    return torch.where(sign == 1, -value, value).double()


def q4_weights(codes, scales, k, group):
    return q4_values(codes, k) * scales.double()[:, torch.arange(k, device=codes.device) // group]


def q4_forward(x, codes, scales, bias, k, group, relu):
    z = x.double() @ q4_weights(codes, scales, k, group).t().contiguous()
    if bias is not None:
        z = z + bias.double()
    return z.clamp(min=0.0) if relu else z

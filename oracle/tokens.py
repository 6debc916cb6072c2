"""Oracle for the operators of a policy over tokens (include/mi355lp.h, mi355gn.h, mi355q4.h, mi355sm.h,
mi355i8.h) -- TEST INFRASTRUCTURE ONLY: torch
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


def kept_weights(row, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row's weights relative to its largest logit, 0 where a limit leaves the token out; None where there is nothing to draw from.
    Token by token, as the limits are defined."""
    x = [float(v) + 0.0 for v in row.double().tolist()]
    top = max(x)
    if not all(v < math.inf for v in x) or top == -math.inf:
        return None
    w = [math.exp(scale * (v - top)) for v in x]
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p < 1.0:
        whole, reached, n = math.fsum(w[i] for i in order), 0.0, 0
        while n < len(order) and (n == 0 or reached < top_p * whole):
            reached = math.fsum((reached, w[order[n]]))
            n += 1
        order = order[:n]
    kept = {i for i in order if min_p <= 0 or w[i] >= min(min_p, 1.0)}
    return [w[i] if i in kept else 0.0 for i in range(len(x))]


def draw_row(row, u, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log probability) of one row, as kept_weights."""
    if not (2.0 ** -60 <= scale <= 2.0 ** 60 and 0.0 <= u <= 1.0) or math.isnan(top_p) or math.isnan(min_p):
        return -1, math.nan
    w = kept_weights(row, scale, top_k, top_p, min_p)
    if w is None:
        return -1, -math.inf if bool((row == -math.inf).all()) else math.nan
    whole, before, last = math.fsum(w), 0.0, 0
    for i, v in enumerate(w):
        if v > 0:
            last = i
            before += v
            if before > u * whole:
                break
    return last, math.log(w[last] / whole)


def draw(logits, u, scale, top_k, top_p, min_p):
    """The same of many long rows, by a sort on the device."""
    x = logits.double() + 0.0
    w = torch.exp(scale.double()[:, None] * (x - x.amax(1, keepdim=True)))
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    place = torch.arange(x.shape[1], device=x.device)[None]
    by = w.gather(1, order)
    by = torch.where((place < top_k[:, None]) | (top_k <= 0)[:, None], by, 0.0)
    sums = by.cumsum(1)
    before = (sums < top_p.double()[:, None] * sums[:, -1:]).sum(1, keepdim=True)
    by = torch.where((place <= before) | (top_p >= 1)[:, None], by, 0.0)
    by = torch.where((by >= min_p.double().clamp(max=1.0)[:, None]) | (min_p <= 0)[:, None], by, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, by)
    sums = w.cumsum(1)
    passed = (sums > u.double()[:, None] * sums[:, -1:]) & (w > 0)
    last = torch.where(w > 0, place, -1).amax(1)
    token = torch.where(passed.any(1), passed.int().argmax(1), last)
    return token.int(), torch.log(w.gather(1, token[:, None])[:, 0] / sums[:, -1])


def eight_bits(x):
    """(codes, scales) of rows in 8 bits, in double: the scale by looking for it."""
    bad = ~torch.isfinite(x.double()).all(1)
    scales = []
    for most in torch.where(bad, 1.0, x.double().abs().amax(1)).tolist():
        unit = math.ldexp(1.0, math.frexp(most)[1] - 20) if most else 1.0
        scale = 0.0
        while most and not scale:  # 128 to 255 of a power of two: the first power that has one which reaches
            if 127 * 255 * unit >= most:
                scale = min(c * unit for c in range(128, 256) if 127 * c * unit >= most)
            unit *= 2.0
        scales.append(max(scale, 2.0 ** -126))
    scale = torch.tensor(scales, dtype=torch.float64, device=x.device)
    codes = torch.round(torch.where(bad[:, None], torch.zeros_like(x, dtype=torch.float64), x.double()) / scale[:, None])
    return codes, torch.where(bad, torch.full_like(scale, math.nan), scale)


def i8_forward(codes, scale, w_codes, w_scale, bias, relu):
    z = (codes.double() @ w_codes.double().t().contiguous()) * scale.double()[:, None] * w_scale.double()[None]
    if bias is not None:
        z = z + bias.double()
    return torch.where(z > 0, z, torch.zeros_like(z)) if relu else z


def i8_backward_filter(codes, scale, dz):
    return (dz.double() * scale.double()[:, None]).t().contiguous() @ codes.double(), dz.double().sum(0)


def i8_backward_data(w_codes, w_scale, dz):
    return (dz.double() * w_scale.double()[None]) @ w_codes.double()

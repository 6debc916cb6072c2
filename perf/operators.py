"""The work of a policy over tokens whose time counts: log probabilities of given tokens with their entropy and top
alternatives, the gradient of a loss on them, clipping by the global gradient norm, and the InnerProduct layer on 4-bit weights.

``run`` computes a case in its plain form from elementary operations, or, where ``own`` is set, through the
framework's entry points.  Sizes are those of vocabularies and layers in common use and of the repository's own layers;
``draw`` spreads them over the ranges that the listed cases stand for.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f64": torch.float64}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "f64": 8}
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)  # the 4-bit floating type


def _tokens(name, kind, rows, vocab, dtype, stride=0, top=0, entropy=1, scale=1.0, masked=0):
    """kind: "score" (log probabilities, entropy, alternatives), "train" (log probabilities, entropy and the gradient of a loss
    whose weights are known before the call) or "grad" (the gradient alone, on a row's statistics from an earlier call)."""
    return dict(name=name, kind=kind, rows=rows, vocab=vocab, dtype=dtype, stride=stride or vocab, top=top, entropy=entropy,
                scale=scale, masked=masked)


def _clip(name, layers, width, vocab, dtype, ratio, inplace, odd=0):
    """Gradients of `layers` blocks of a network `width` wide under an embedding of `vocab` rows.  ratio: the limit over the norm
    that is expected.  odd: sizes that are multiples of nothing, from the second element of a buffer on, every fifth tensor in
    another type.  A step that does not clip may run in place, again and again; one that clips writes to other buffers."""
    return dict(name=name, kind="clip", layers=layers, width=width, vocab=vocab, dtype=dtype, ratio=ratio, inplace=inplace, odd=odd)


def _matvec(name, m, k, o, dtype, group, bias=0, relu=0):
    return dict(name=name, kind="matvec", m=m, k=k, o=o, dtype=dtype, group=group, bias=bias, relu=relu)


def listed():
    return [
        # one token being generated: its log probability and twenty alternatives; latency counts
        _tokens("score_one", "score", 1, 32000, "bf16", top=20),
        # a step of generation for a batch of 64 on a large vocabulary
        _tokens("score_batch", "score", 64, 128256, "bf16", top=20),
        # scoring given texts: odd vocabulary in padded rows, banned tokens, another temperature
        _tokens("score_texts", "score", 777, 50257, "f16", stride=50304, top=5, scale=1.25, masked=1),
        # policy gradient on the repository's thousand-output layer, fp32
        _tokens("train_thousand", "train", 512, 1000, "f32", entropy=0),
        # policy gradient with an entropy bonus on a large vocabulary: the largest
        _tokens("train_large", "train", 4096, 128256, "bf16"),
        # the gradient where the weights depend on the log probabilities (ratios to an older policy)
        _tokens("grad_ratio", "grad", 2048, 50257, "bf16", masked=1),
        # a digit-sized network's gradients, step after step without clipping
        _clip("clip_small", 4, 64, 200, "f32", 4.0, 1),
        # a language model's bf16 gradients, clipped
        _clip("clip_large", 24, 1024, 50304, "bf16", 0.25, 0),
        # sizes that are multiples of nothing, views of one buffer, two types
        _clip("clip_odd", 10, 517, 9999, "f32", 0.5, 0, odd=1),
        # one token through a square layer
        _matvec("token_square", 1, 4096, 4096, "bf16", 128),
        # one token to the logits of a large vocabulary
        _matvec("token_logits", 1, 4096, 128256, "bf16", 32),
        # a batch through the repository's widest fully connected layer
        _matvec("batch_fc", 48, 9216, 4096, "f32", 64, bias=1, relu=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    while True:
        r = rng.random()
        if r < 0.6:
            kind = "score" if r < 0.3 else "train" if r < 0.48 else "grad"
            rows, vocab = _log_int(rng, 1, 8192), _log_int(rng, 64, 160000)
            if rng.random() < 0.3:
                vocab = vocab // 8 * 8
            if rows * vocab > 4096 * 100000:
                continue
            case = _tokens("", kind, rows, vocab, rng.choice(("bf16", "bf16", "f16", "f32")),
                           stride=vocab + (rng.randrange(64) if rng.random() < 0.4 else 0),
                           top=min(rng.randint(0, 32), vocab // 2) if kind == "score" else 0,
                           entropy=int(rng.random() < 0.7), scale=rng.choice((1.0, 1.0, 0.75, 1.5)),
                           masked=int(vocab >= 500 and rng.random() < 0.4))
        elif r < 0.78:
            ratio = rng.choice((0.25, 0.6, 4.0))
            case = _clip("", _log_int(rng, 1, 40), _log_int(rng, 8, 1024), _log_int(rng, 10, 50000),
                         rng.choice(("f32", "f32", "bf16", "f16", "f64")), ratio, int(ratio > 1 and rng.random() < 0.5),
                         odd=int(rng.random() < 0.5))
            if sum(_counts(case)) > 2.5e8:
                continue
        else:
            case = _matvec("", _log_int(rng, 1, 64), _log_int(rng, 32, 12288), _log_int(rng, 8, 128256),
                           rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice((32, 64, 128)), bias=rng.randrange(2),
                           relu=int(rng.random() < 0.3))
            if case["k"] * case["o"] > 4096 * 100000 or case["m"] * case["k"] * case["o"] > 48 * 9216 * 4096:
                continue
        del case["name"]
        return case


# ---- log probabilities ----

def _token_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    logits = torch.randn((rows, case["stride"]), generator=g, device=DEV).mul_(2.5)
    token = torch.randint(vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if case["masked"]:  # tokens that the program bans everywhere
        logits.masked_fill_(torch.rand((1, case["stride"]), generator=g, device=DEV) < 0.05, -math.inf)
    at = torch.arange(rows, device=DEV)
    logits[at, token.long()] = torch.randn(rows, generator=g, device=DEV).mul_(2).add_(5)  # what was sampled is likely
    logits = logits.to(TYPES[case["dtype"]])[:, :vocab]
    if case["kind"] != "score":
        token.masked_fill_(torch.rand(rows, generator=g, device=DEV) < 0.03, -1)  # positions that count for nothing
    d_logp = torch.randn(rows, generator=g, device=DEV) / rows
    d_entropy = torch.full((rows,), -0.01 / rows, device=DEV) if case["entropy"] else None
    return logits, token, d_logp, d_entropy


def _token_state(case, seed):
    s = dict(case=case)
    s["logits"], s["token"], s["d_logp"], s["d_entropy"] = _token_inputs(case, seed)
    if own:
        import paper_1810_02272_amd as lib
        rows, top = case["rows"], case["top"]
        s["desc"] = lib.lp_desc_create(lib.LpParams(rows, case["vocab"], TYPES[case["dtype"]], top, case["entropy"], case["scale"]))
        s["ws"] = torch.empty(max(lib.lp_desc_workspace_bytes(s["desc"]) // 4, 1), device=DEV)
        s["logp"], s["stats"] = torch.empty(rows, device=DEV), torch.empty((rows, 4), device=DEV)
        s["h"] = torch.empty(rows, device=DEV) if case["entropy"] else None
        s["top_logp"] = torch.empty((rows, top), device=DEV) if top else None
        s["top_token"] = torch.empty((rows, top), device=DEV, dtype=torch.int32) if top else None
        if case["kind"] != "score":
            s["d_logits"] = torch.empty((rows, case["vocab"]), device=DEV, dtype=TYPES[case["dtype"]])
        if case["kind"] == "grad":
            lib.lp_forward(s["desc"], s["logits"], s["token"], s["logp"], s["h"], s["stats"], None, None, s["ws"])
    return s


def _token_own(s):
    import paper_1810_02272_amd as lib
    case = s["case"]
    if case["kind"] == "grad":
        lib.lp_backward(s["desc"], s["logits"], s["token"], s["stats"], s["d_logp"], s["d_entropy"], s["d_logits"])
        return [s["d_logits"]]
    if case["kind"] == "train":
        lib.lp_forward_backward(s["desc"], s["logits"], s["token"], s["d_logp"], s["d_entropy"], s["logp"], s["h"], s["d_logits"], s["ws"])
        return [s["logp"], s["h"], s["d_logits"]] if case["entropy"] else [s["logp"], s["d_logits"]]
    lib.lp_forward(s["desc"], s["logits"], s["token"], s["logp"], s["h"], None, s["top_logp"], s["top_token"], s["ws"])
    return [t for t in (s["logp"], s["h"], s["top_logp"], s["top_token"]) if t is not None]


def _token_plain(s):
    case, logits, token = s["case"], s["logits"], s["token"]
    z = logits.float() * case["scale"]
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    at = token.long().clamp(min=0)[:, None]
    logp = torch.where(token >= 0, (d.gather(1, at) - log_total)[:, 0], 0.0)
    out, h = [logp], None
    if case["entropy"]:
        h = log_total - (torch.where(e > 0, d, 0.0) * e).sum(1, keepdim=True) / total
        out.append(h[:, 0])
    if case["kind"] == "score":
        if case["top"]:
            value, index = torch.sort(logits, dim=1, descending=True, stable=True)
            value, index = value[:, :case["top"]], index[:, :case["top"]]
            out += [value.float() * case["scale"] - m - log_total, index.int()]
        return out
    p = e / total
    g = -s["d_logp"][:, None] * (token >= 0)[:, None] * p
    g.scatter_add_(1, at, torch.where(token >= 0, s["d_logp"], 0.0)[:, None])
    if case["entropy"]:
        g -= s["d_entropy"][:, None] * p * (torch.where(e > 0, d, 0.0) - log_total + h)
    d_logits = (g * case["scale"]).to(logits.dtype)
    return [d_logits] if case["kind"] == "grad" else out + [d_logits]


def _token_exact(case, seed):
    logits, token, d_logp, d_entropy = _token_inputs(case, seed)
    parts = []
    for rows in torch.arange(case["rows"], device=DEV).split(max(1, int(1.5e8) // case["vocab"])):
        z = logits[rows].double() * case["scale"]
        logq = z - torch.logsumexp(z, 1, keepdim=True)
        q = logq.exp()
        h = -torch.xlogy(q, q).sum(1)
        valid = (token[rows] >= 0).double()
        at = token[rows].long().clamp(min=0)[:, None]
        first = [logq.gather(1, at)[:, 0] * valid] + ([h] if case["entropy"] else [])
        if case["kind"] == "score":
            parts.append(first + ([torch.topk(logq, case["top"], 1).values] if case["top"] else []))
            continue
        w = (d_logp[rows].double() * valid)[:, None]
        g = torch.zeros_like(q).scatter_(1, at, w) - w * q
        if case["entropy"]:
            g -= d_entropy[rows].double()[:, None] * (torch.xlogy(q, q) + q * h[:, None])
        parts.append(([] if case["kind"] == "grad" else first) + [g * case["scale"]])
    out = [torch.cat(p) for p in zip(*parts)]
    return out + [None] if case["kind"] == "score" and case["top"] else out


# ---- clipping ----

def _counts(case):
    w, odd = case["width"], case["odd"]
    block = (w * w + odd, w * w + 2 * odd, w * w, w * w + 5 * odd, 4 * w * w + 3 * odd, 4 * w * w + odd, 4 * w + odd, w, w + odd, w)
    return [case["vocab"] * w + odd] + list(block) * case["layers"] + [w]


def _clip_types(case):
    n = 2 + 10 * case["layers"]
    other = "bf16" if case["dtype"] != "bf16" else "f32"
    return [other if case["odd"] and i % 5 == 4 else case["dtype"] for i in range(n)]


def _buckets(case, fill):
    """One buffer for each type: its tensors follow each other in it, where `odd` from its second element on."""
    size = dict.fromkeys(sorted(set(_clip_types(case))), case["odd"])
    for n, t in zip(_counts(case), _clip_types(case)):
        size[t] += n
    return {t: fill(n, TYPES[t]) for t, n in size.items()}


def _views(case, buckets):
    at, out = dict.fromkeys(buckets, case["odd"]), []
    for n, t in zip(_counts(case), _clip_types(case)):
        out.append(buckets[t][at[t]:at[t] + n])
        at[t] += n
    return out


def _gradients(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return _buckets(case, lambda n, t: torch.randn(n, generator=g, device=DEV).to(t))


def _limit(case):
    return case["ratio"] * math.sqrt(sum(_counts(case)))


def _clip_state(case, seed):
    s = dict(case=case, buckets=_gradients(case, seed), limit=_limit(case))
    if own:
        import paper_1810_02272_amd as lib
        s["out_buckets"] = s["buckets"] if case["inplace"] else _buckets(case, lambda n, t: torch.empty(n, device=DEV, dtype=t))
        s["grads"], s["outs"] = _views(case, s["buckets"]), _views(case, s["out_buckets"])
        s["desc"] = lib.gn_desc_create(lib.GnParams([t.numel() for t in s["grads"]], [t.dtype for t in s["grads"]]))
        s["ws"] = torch.empty(max(lib.gn_desc_workspace_bytes(s["desc"]) // 4, 1), device=DEV)
        s["norm"] = torch.empty(1, device=DEV)
    return s


def _clip_own(s):
    import paper_1810_02272_amd as lib
    lib.gn_clip(s["desc"], s["grads"], s["limit"], s["outs"], s["norm"], s["ws"])
    return [s["norm"]] + [b[s["case"]["odd"]:] for b in s["out_buckets"].values()]


def _clip_plain(s):  # a buffer's tensors need not be told apart: the sum runs over all of them, and one factor goes to all
    grads = [b[s["case"]["odd"]:] for b in s["buckets"].values()]
    norm = torch.stack([t.double().square().sum() for t in grads]).sum().sqrt()
    scale = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm))
    return [norm.float().view(1)] + [(t * scale if t.dtype == torch.float64 else t.float() * scale.float()).to(t.dtype) for t in grads]


def _clip_exact(case, seed):
    grads = [b[case["odd"]:].double() for b in _gradients(case, seed).values()]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t) for t in grads]))
    factor = min(1.0, _limit(case) / float(norm))
    return [norm.view(1)] + [t * factor for t in grads]


# ---- 4-bit weights ----

def _matvec_inputs(case, seed):
    """x, the codes two a byte (the first in the low half), the scales, the bias."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m, k, o, group, t = case["m"], case["k"], case["o"], case["group"], TYPES[case["dtype"]]
    x = torch.randn((m, k), generator=g, device=DEV).to(t)
    groups = -(-k // group)
    scales = (torch.rand((o, groups), generator=g, device=DEV).add_(0.5).mul_(1.0 / math.sqrt(8.0 * k))).to(torch.bfloat16)
    codes = torch.randint(256, (o, (k + 1) // 2), generator=g, device=DEV, dtype=torch.uint8)
    if k % 2:
        codes[:, -1] &= 15
    bias = torch.randn(o, generator=g, device=DEV).to(t) if case["bias"] else None
    return x, codes, scales, bias


def _matvec_state(case, seed):
    s = dict(case=case)
    s["x"], s["codes"], s["scales"], s["bias"] = _matvec_inputs(case, seed)
    if own:
        import paper_1810_02272_amd as lib
        s["desc"] = lib.q4_desc_create(lib.Q4Params(case["m"], case["k"], case["o"], TYPES[case["dtype"]], case["group"], case["bias"], case["relu"]))
        s["packed"] = torch.empty(lib.q4_desc_packed_bytes(s["desc"]), device=DEV, dtype=torch.uint8)
        lib.q4_pack(s["desc"], s["codes"], s["scales"], s["packed"])
        s["ws"] = torch.empty(max(lib.q4_desc_workspace_bytes(s["desc"]) // 4, 1), device=DEV)
        s["y"] = torch.empty((case["m"], case["o"]), device=DEV, dtype=TYPES[case["dtype"]])
    return s


def _matvec_own(s):
    import paper_1810_02272_amd as lib
    lib.q4_forward(s["desc"], s["x"], s["packed"], s["bias"], s["y"], s["ws"])
    return [s["y"]]


def _weights(case, codes, scales, dtype):
    both = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1)[:, :case["k"]]
    return torch.tensor(CODES, device=DEV, dtype=dtype)[both.int()] * scales.to(dtype).repeat_interleave(case["group"], 1)[:, :case["k"]]


def _matvec_plain(s):
    case = s["case"]
    y = s["x"].float() @ _weights(case, s["codes"], s["scales"], torch.float32).t()
    if case["bias"]:
        y += s["bias"].float()
    if case["relu"]:
        y = torch.where(y > 0, y, 0.0)
    return [y.to(s["x"].dtype)]


def _matvec_exact(case, seed):
    x, codes, scales, bias = _matvec_inputs(case, seed)
    per = max(1, int(1e8) // case["k"])
    value = torch.tensor([v for c in range(256) for v in (CODES[c % 16], CODES[c // 16])], device=DEV, dtype=torch.float64).view(256, 2)
    parts = []
    for c, sc in zip(codes.split(per), scales.split(per)):
        w = value[c.int()].view(c.shape[0], -1)[:, :case["k"]]
        group = torch.arange(case["k"], device=DEV) // case["group"]
        parts.append(x.double() @ (w * sc.double()[:, group]).t())
    y = torch.cat(parts, 1)
    if bias is not None:
        y = y + bias.double()
    return [y.clamp(min=0.0) if case["relu"] else y]


# ---- what is measured ----

def prepare(case, seed):
    return _clip_state(case, seed) if case["kind"] == "clip" else _matvec_state(case, seed) if case["kind"] == "matvec" else _token_state(case, seed)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _clip_own(state) if kind == "clip" else _matvec_own(state) if kind == "matvec" else _token_own(state)
    return _clip_plain(state) if kind == "clip" else _matvec_plain(state) if kind == "matvec" else _token_plain(state)


def exact(case, seed):
    kind = case["kind"]
    return _clip_exact(case, seed) if kind == "clip" else _matvec_exact(case, seed) if kind == "matvec" else _token_exact(case, seed)


def work(case):
    if case["kind"] == "clip":
        counts, types = _counts(case), _clip_types(case)
        read = sum(n * SIZE[t] for n, t in zip(counts, types))
        return {"bytes": read * (1 if case["inplace"] else 2), "flops": 3.0 * sum(counts)}
    if case["kind"] == "matvec":
        m, k, o = case["m"], case["k"], case["o"]
        size = SIZE[case["dtype"]]
        return {"bytes": o * ((k + 1) // 2 + 2 * -(-k // case["group"])) + size * (m * k + m * o + o * case["bias"]), "flops": 2.0 * m * k * o}
    n = case["rows"] * case["vocab"]
    read = n * SIZE[case["dtype"]]
    a_row = 4 + (4 + 4 * case["entropy"] if case["kind"] != "grad" else 0) + 8 * case["top"] + (4 + 4 * case["entropy"] if case["kind"] != "score" else 0)
    return {"bytes": read * (1 if case["kind"] == "score" else 2) + a_row * case["rows"], "flops": (5.0 if case["kind"] == "score" else 8.0) * n}

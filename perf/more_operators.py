"""More work of a policy over tokens whose time counts: drawing tokens under temperature, top-k, top-p and min-p, the InnerProduct
layer in 8-bit integers with a scale for each token and channel, and its gradients from activations kept in 8 bits.

``run`` computes a case in its plain form from elementary operations, or, where ``own`` is set, through the
framework's entry points.  Sizes are those of vocabularies and layers in common use and of the repository's own layers;
``draw`` spreads them over the ranges that the listed cases stand for.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _draws(name, rows, vocab, dtype, stride=0, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=0, masked=0, spread=1.5):
    """mixed: every row has parameters of its own, some of them none.  spread: of the logits around their ranks' share."""
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, stride=stride or vocab, scale=scale, top_k=top_k,
                top_p=top_p, min_p=min_p, mixed=mixed, masked=masked, spread=spread)


def _layer(name, kind, m, k, o, dtype, bias=0, relu=0):
    """kind: "forward" (rows to 8 bits, their product with weights in 8 bits), "filter" (rows kept in 8 bits, and the gradients of
    weights and bias from them) or "data" (the rows' gradient from weights in 8 bits)."""
    return dict(name=name, kind=kind, m=m, k=k, o=o, dtype=dtype, bias=bias, relu=relu)


def listed():
    return [
        # one token being generated with the usual three limits; latency counts
        _draws("sample_one", 1, 32000, "bf16", scale=1.25, top_k=50, top_p=0.9),
        # a step of generation for a batch of 64 on a large vocabulary
        _draws("sample_batch", 64, 128256, "bf16", top_p=0.95, min_p=0.01),
        # requests of different settings in one batch: odd vocabulary in padded rows, banned tokens
        _draws("sample_mixed", 333, 50257, "f16", stride=50304, mixed=1, masked=1),
        # playing many episodes at once, temperature alone
        _draws("sample_rollout", 1024, 128256, "bf16", scale=0.75),
        # one token through a square layer
        _layer("token_square", "forward", 1, 4096, 4096, "bf16"),
        # a batch through the repository's widest fully connected layer
        _layer("batch_fc", "forward", 48, 9216, 4096, "f32", bias=1, relu=1),
        # a whole prompt through a square layer: the largest
        _layer("prompt_square", "forward", 8192, 4096, 4096, "bf16"),
        # the repository's thousand-output layer, trained in fp32
        _layer("filter_thousand", "filter", 256, 4096, 1000, "f32", bias=1),
        # a training step's weight gradient, bf16
        _layer("filter_square", "filter", 8192, 4096, 4096, "bf16"),
        # sizes that are multiples of nothing
        _layer("filter_odd", "filter", 1999, 1111, 777, "f16", bias=1),
        # a training step's input gradient, bf16
        _layer("data_square", "data", 8192, 4096, 4096, "bf16"),
        # a small layer's, odd
        _layer("data_odd", "data", 100, 999, 333, "f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    while True:
        if rng.random() < 0.5:
            rows, vocab = _log_int(rng, 1, 4096), _log_int(rng, 16, 160000)
            if rng.random() < 0.3 and vocab >= 64:
                vocab = vocab // 8 * 8
            if rows * vocab > 1024 * 128000:
                continue
            case = _draws("", rows, vocab, rng.choice(("bf16", "bf16", "f16", "f32")),
                          stride=vocab + (rng.randrange(64) if rng.random() < 0.4 else 0), scale=rng.choice((1.0, 0.5, 0.75, 1.25, 2.0)),
                          top_k=rng.choice((0, 0, 1, 20, 50, 1000)), top_p=rng.choice((1.0, 1.0, 0.5, 0.9, 0.95, 0.99)),
                          min_p=rng.choice((0.0, 0.0, 0.01, 0.05, 0.2)), mixed=int(rng.random() < 0.3),
                          masked=int(vocab >= 500 and rng.random() < 0.4), spread=rng.choice((0.5, 1.5, 1.5, 3.0)))
        else:
            kind = rng.choice(("forward", "filter", "data"))
            case = _layer("", kind, _log_int(rng, 1, 8192), _log_int(rng, 16, 12288), _log_int(rng, 8, 16384),
                          rng.choice(("bf16", "bf16", "f16", "f32")), bias=rng.randrange(2) if kind != "data" else 0,
                          relu=int(kind == "forward" and rng.random() < 0.3))
            if case["m"] * case["k"] * case["o"] > 8192 * 4096 * 2048 or case["k"] * case["o"] > 1e8:
                continue
        del case["name"]
        return case


# ---- drawing tokens ----

def _sample_inputs(case, seed):
    """logits, uniform numbers, and the rows' scale, top_k, top_p and min_p."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    logits = torch.empty((rows, case["stride"]), device=DEV, dtype=TYPES[case["dtype"]])
    banned = torch.rand((1, case["stride"]), generator=g, device=DEV) < 0.05
    for part in logits.split(256):
        # a few tokens are likely and most are not: a share that falls with a random rank, and noise
        z = torch.rand(part.shape, generator=g, device=DEV).mul_(vocab).add_(1.0).log_().mul_(-1.2)
        z.add_(torch.randn(part.shape, generator=g, device=DEV), alpha=case["spread"]).add_(12.0)
        if case["masked"]:
            z.masked_fill_(banned, -math.inf)
        part.copy_(z)
    if case["masked"]:
        logits[:, vocab // 2] = 3.0  # one is always allowed
    u = torch.rand(rows, generator=g, device=DEV)
    full = lambda v, t=torch.float32: torch.full((rows,), v, device=DEV, dtype=t)
    scale, top_k, top_p, min_p = full(case["scale"]), full(case["top_k"], torch.int32), full(case["top_p"]), full(case["min_p"])
    if case["mixed"]:
        pick = lambda values, t=torch.float32: torch.tensor(values, device=DEV, dtype=t)[torch.randint(len(values), (rows,), generator=g, device=DEV)]
        scale, top_k = pick((0.5, 0.75, 1.0, 1.25, 2.0)), pick((0, 0, 1, 5, 40, 200, 3000), torch.int32)
        top_p, min_p = pick((1.0, 0.3, 0.8, 0.9, 0.95, 0.99)), pick((0.0, 0.0, 0.02, 0.1))
    return logits[:, :vocab], u, scale, top_k, top_p, min_p


def _sample_state(case, seed):
    s = dict(case=case)
    s["logits"], s["u"], s["scale"], s["top_k"], s["top_p"], s["min_p"] = _sample_inputs(case, seed)
    if own:
        import paper_1810_02272_amd as lib
        if not case["mixed"]:  # a limit that no row has is not given
            s["top_k"] = s["top_k"] if case["top_k"] else None
            s["top_p"] = s["top_p"] if case["top_p"] < 1 else None
            s["min_p"] = s["min_p"] if case["min_p"] else None
        s["desc"] = lib.sm_desc_create(lib.SmParams(case["rows"], case["vocab"], TYPES[case["dtype"]]))
        s["ws"] = torch.empty(max(lib.sm_desc_workspace_bytes(s["desc"]) // 4, 1), device=DEV)
        s["token"], s["logp"] = torch.empty(case["rows"], device=DEV, dtype=torch.int32), torch.empty(case["rows"], device=DEV)
    return s


def _sample_own(s):
    import paper_1810_02272_amd as lib
    lib.sm_sample(s["desc"], s["logits"], s["u"], s["scale"], s["top_k"], s["top_p"], s["min_p"], s["token"], s["logp"], s["ws"])
    return [s["token"], s["logp"]]


def _limits(x, scale, top_k, top_p, min_p, ordered):
    """Weights of the logits in 64 bits, 0 where a limit leaves a token out."""
    most = x.amax(1, keepdim=True).double()
    w = torch.exp((x.double() - most) * scale.double()[:, None])
    if not ordered:  # no limit by order
        return torch.where(w >= min_p.double().clamp(max=1.0)[:, None], w, 0.0)
    index = torch.sort(x, dim=1, descending=True, stable=True)[1]
    place = torch.arange(x.shape[1], device=DEV)
    by = w.gather(1, index)
    k = torch.where(top_k > 0, top_k, x.shape[1])[:, None]
    by = torch.where(place < k, by, 0.0)
    sums = by.cumsum(1)
    reached = (sums < top_p.double()[:, None] * sums[:, -1:]).sum(1, keepdim=True)  # those before the one that reaches it
    keep = (by >= min_p.double().clamp(max=1.0)[:, None]) & ((place <= reached) | (top_p >= 1.0)[:, None])
    return torch.zeros_like(w).scatter_(1, index, torch.where(keep, by, 0.0))


def _sample_plain(s):
    case = s["case"]
    ordered = bool(case["mixed"] or case["top_k"] or case["top_p"] < 1)
    token, logp = [], []
    per = max(1, int(6e7) // case["vocab"])
    for first in range(0, case["rows"], per):
        at = slice(first, first + per)
        w = _limits(s["logits"][at], s["scale"][at], s["top_k"][at], s["top_p"][at], s["min_p"][at], ordered)
        sums = w.cumsum(1)
        total = sums[:, -1:]
        last = w.shape[1] - 1
        t = (sums <= s["u"][at].double()[:, None] * total).sum(1, keepdim=True).clamp(max=last)
        token.append(t[:, 0].int())
        logp.append(torch.log(w.gather(1, t) / total)[:, 0].float())
    return [torch.cat(token), torch.cat(logp)]


def _sample_exact(case, seed):
    """Row by row: the tokens that are kept, in the order of their indices, and the one that the uniform number falls on; its log probability."""
    logits, u, scale, top_k, top_p, min_p = _sample_inputs(case, seed)
    out = []
    for r in range(case["rows"]):
        index = torch.sort(logits[r], descending=True, stable=True).indices
        z = (logits[r].double() - logits[r][index[0]].double()) * scale[r].double()
        n = int(top_k[r]) if 0 < int(top_k[r]) < case["vocab"] else case["vocab"]
        chosen = index[:n]
        if float(top_p[r]) < 1.0:
            p = z[chosen].exp().cumsum(0)
            chosen = chosen[:int(torch.searchsorted(p, top_p[r].double() * p[-1])) + 1]
        if float(min_p[r]) > 0.0:
            chosen = chosen[z[chosen] >= math.log(min(float(min_p[r]), 1.0))]
        chosen = chosen.sort().values
        p = z[chosen].exp().cumsum(0)
        place = min(int(torch.searchsorted(p, u[r].double() * p[-1], right=True)), len(chosen) - 1)
        out.append(z[chosen][place] - p[-1].log())
    return [None, torch.stack(out)]


# ---- a layer in 8 bits ----

def _layer_inputs(case, seed):
    """x, w, bias, and the gradient of the outputs."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m, k, o, t = case["m"], case["k"], case["o"], TYPES[case["dtype"]]
    random = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    x = random(m, k).mul_(random(m, 1).mul_(0.5).exp_())  # tokens of different sizes
    x[:, random(k) > 2.5] *= 6.0  # and inputs that stand out
    w = random(o, k).mul_(random(o, 1).mul_(0.3).exp_()).div_(math.sqrt(k))
    return x.to(t), w.to(t), random(o).to(t), random(m, o).div_(m).to(t)


def _eight(x):
    """Codes as 32-bit numbers, and the scales: the smallest of 8 significant bits whose 127-fold reaches a row's largest magnitude."""
    most = x.float().abs().amax(1, keepdim=True)
    down = ((most / 127.0).view(torch.int32) & -65536).view(torch.float32)
    up = ((most / 127.0).view(torch.int32) + 65536 & -65536).view(torch.float32)
    scale = torch.where(down * 127.0 >= most, down, up).clamp(min=2.0 ** -126)
    return torch.round(x.double() / scale.double()).float(), scale


def _layer_state(case, seed):
    x, w, bias, dz = _layer_inputs(case, seed)
    s = dict(case=case, dz=dz, bias=bias if case["bias"] else None, x=x)
    if case["kind"] != "filter":  # weights are laid out once
        if not own:
            s["w_codes"], s["w_scale"] = _eight(w)
    if own:
        import paper_1810_02272_amd as lib
        m, k, o, t = case["m"], case["k"], case["o"], TYPES[case["dtype"]]
        f = lambda *shape, dtype=torch.float32: torch.empty(shape, device=DEV, dtype=dtype)
        d = s["desc"] = lib.i8_desc_create(lib.I8Params(m, k, o, t, case["bias"], case["relu"]))
        row = lib.i8_desc_row_bytes(d)
        s["ws"] = f(max(lib.i8_desc_workspace_bytes(d) // 4, 1))
        s["codes"], s["scale"] = f(m, row, dtype=torch.int8), f(m)
        if case["kind"] != "filter":
            s["w_codes"], s["w_scale"] = f(o, row, dtype=torch.int8), f(o)
            lib.i8_pack(d, w, s["w_codes"], s["w_scale"])
        s["y"] = f(m, o, dtype=t) if case["kind"] == "forward" else None
        s["dx"] = f(m, k, dtype=t) if case["kind"] == "data" else None
        if case["kind"] == "filter":
            s["dw"], s["db"] = f(o, k), f(o) if case["bias"] else None
    return s


def _layer_own(s):
    import paper_1810_02272_amd as lib
    kind = s["case"]["kind"]
    if kind == "forward":
        lib.i8_forward(s["desc"], s["x"], s["w_codes"], s["w_scale"], s["bias"], s["y"], s["codes"], s["scale"], s["ws"])
        return [s["y"]]
    if kind == "data":
        lib.i8_backward_data(s["desc"], s["w_codes"], s["w_scale"], s["dz"], s["dx"], s["ws"])
        return [s["dx"]]
    lib.i8_quantise(s["desc"], s["x"], s["codes"], s["scale"])
    lib.i8_backward_filter(s["desc"], s["codes"], s["scale"], s["dz"], s["dw"], s["db"], 0.0, s["ws"])
    return [t for t in (s["dw"], s["db"]) if t is not None]


def _layer_plain(s):
    case = s["case"]
    if case["kind"] == "forward":
        codes, scale = _eight(s["x"])
        y = (codes @ s["w_codes"].t()) * (scale * s["w_scale"].t())
        if case["bias"]:
            y += s["bias"].float()
        return [(torch.where(y > 0, y, 0.0) if case["relu"] else y).to(s["x"].dtype)]
    if case["kind"] == "data":
        return [((s["dz"].float() * s["w_scale"].t()) @ s["w_codes"]).to(s["dz"].dtype)]
    codes, scale = _eight(s["x"])
    out = [(s["dz"].float() * scale).t() @ codes]
    return out + [s["dz"].double().sum(0).float()] if case["bias"] else out


def _values(x):
    """What rows stand for in 8 bits, in 64 bits."""
    most = x.double().abs().amax(1, keepdim=True)
    fraction, exponent = torch.frexp(most / torch.full_like(most, 127.0))  # (a number's reciprocal would be taken)
    scale = torch.ceil(fraction * 256.0) * (exponent.long() + (1023 - 8) << 52).view(torch.float64)
    scale = scale.clamp(min=2.0 ** -126)
    return torch.round(x.double() / scale) * scale


def _layer_exact(case, seed):
    x, w, bias, dz = _layer_inputs(case, seed)
    if case["kind"] == "forward":
        y = _values(x) @ _values(w).t()
        if case["bias"]:
            y = y + bias.double()
        return [y.clamp(min=0.0) if case["relu"] else y]
    if case["kind"] == "data":
        return [dz.double() @ _values(w)]
    out = [dz.double().t() @ _values(x)]
    return out + [dz.double().sum(0)] if case["bias"] else out


# ---- what is measured ----

def prepare(case, seed):
    return _sample_state(case, seed) if case["kind"] == "sample" else _layer_state(case, seed)


def run(state):
    if state["case"]["kind"] == "sample":
        return _sample_own(state) if own else _sample_plain(state)
    return _layer_own(state) if own else _layer_plain(state)


def exact(case, seed):
    return _sample_exact(case, seed) if case["kind"] == "sample" else _layer_exact(case, seed)


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZE[case["dtype"]] + 28 * case["rows"], "flops": 16.0 * n}
    m, k, o, size = case["m"], case["k"], case["o"], SIZE[case["dtype"]]
    read = {"forward": size * m * k + o * k + 4 * o, "filter": size * (m * k + m * o), "data": size * m * o + o * k + 4 * o}[case["kind"]]
    written = {"forward": size * m * o, "filter": 4 * o * k, "data": size * m * k}[case["kind"]]
    return {"bytes": read + written + case["bias"] * o * (size if case["kind"] == "forward" else 4), "flops": 2.0 * m * k * o}

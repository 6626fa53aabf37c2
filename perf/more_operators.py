"""The operators of the 8-bit decoder path whose speed this framework is held
to, with the sizes and value distributions they meet in use.

A case is one call (or the calls of one step of a serving program):

  op "matmul"   w8_matmul: rows times a weight matrix in 8-bit integers, with a
                scale for each row and each output; with `step` after a
                w8_quantize of 16-bit rows, as a layer calls them
  op "route"    route_experts: which experts a token goes to, with what weights,
                and the tokens in the order of their experts
  op "experts"  w8_experts_matmul: each route's product with its expert's
                weights; with `combine` the weighted sum of a token's routes

8-bit values: a row's scale is max|x| / 127; a code is 127 x / max|x| rounded
to the nearest integer, halves up.  All zeros: scale 0.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------- the cases

def _matmul(name, m, n, k, dtype, bias=False, step=False):
    c = dict(op="matmul", m=m, n=n, k=k, dtype=dtype, bias=bias, step=step)
    return dict(name=name, **c) if name else c


def _route(name, tokens, experts, top, score, bias, groups, top_groups, group_best, dtype):
    c = dict(op="route", tokens=tokens, experts=experts, top=top, score=score, bias=bias, groups=groups,
             top_groups=top_groups, group_best=group_best, dtype=dtype)
    return dict(name=name, **c) if name else c


def _experts(name, tokens, experts, top, n, k, dtype, combine=False):
    c = dict(op="experts", tokens=tokens, experts=experts, top=top, n=n, k=k, dtype=dtype, combine=combine)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token through a projection, its activations quantized first: latency
        _matmul("linear_token", 1, 4096, 4096, "bf16", step=True),
        # a prompt through the projection back, long sums, quantized first
        _matmul("linear_prompt", 2048, 4096, 16384, "fp16", step=True),
        # a decoding batch through a feed-forward layer's wide projection
        _matmul("matmul_batch", 48, 16384, 4096, "bf16"),
        # a short prompt, an odd row count (a vocabulary slice), bias
        _matmul("matmul_odd_bias", 333, 5003, 2080, "bf16", bias=True),
        # packed prompts through the wide projection: the matrix cores bound it
        _matmul("matmul_prompt", 8192, 16384, 4096, "bf16"),
        # a decoding batch's routes, few experts: the smallest call, all latency
        _route("route_step", 32, 64, 4, "softmax", False, 1, 1, 1, "bf16"),
        # packed prompts, many experts in groups, balanced by a bias
        _route("route_prompt", 16384, 256, 8, "sigmoid", True, 8, 4, 2, "fp32"),
        # one token to its experts and back: latency
        _experts("experts_token", 1, 8, 2, 1024, 2048, "bf16", combine=True),
        # a decoding batch: nearly every expert's weights are read for a few rows
        _experts("experts_batch", 32, 64, 6, 2816, 2048, "bf16"),
        # a prompt over many small experts, the first product
        _experts("experts_prompt", 4096, 64, 8, 2816, 2048, "bf16"),
        # a prompt over few large experts, the product back with the weighted sum
        _experts("experts_back", 2000, 8, 2, 4096, 8192, "fp16", combine=True),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 8192 rows, 64 to 32768 outputs, sums of
    64 to 16384; 1 to 16384 tokens to 4 to 256 experts; either type."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["matmul", "matmul", "matmul", "route", "experts", "experts"])
    dtype = rng.choice(["bf16", "fp16"])
    while True:
        if op == "matmul":
            c = _matmul(None, log_int(1, 8192), log_int(64, 32768), 16 * log_int(4, 1024), dtype, rng.random() < 0.3,
                        rng.random() < 0.4)
            small = c["m"] * c["n"] * c["k"] <= 1 << 38 and c["n"] * c["k"] <= 1 << 28
        elif op == "route":
            groups, size = rng.choice([1, 1, 2, 4, 8, 16]), rng.choice([2, 3, 4, 8, 16, 32, 60, 64])
            top_groups = rng.randint(max(1, groups // 4), groups)
            c = _route(None, log_int(1, 16384), groups * size, rng.randint(1, min(8, top_groups * size)),
                       rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5, groups, top_groups, rng.choice([1, 2]),
                       rng.choice(["bf16", "fp16", "fp32"]))
            small = 4 <= c["experts"] <= 256
        else:
            e = rng.choice([4, 8, 16, 32, 60, 64, 128])
            c = _experts(None, log_int(1, 8192), e, rng.randint(1, min(8, e)), log_int(64, 8192), 16 * log_int(8, 512),
                         dtype, rng.random() < 0.5)
            small = e * c["n"] * c["k"] <= 1 << 29 and c["tokens"] * c["top"] * c["n"] * c["k"] <= 1 << 37
        if small:
            return c


def work(case):
    c = case
    if c["op"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        x = 2 * m * k + 4 * m if c["step"] else m * k + 4 * m
        return {"bytes": x + n * k + 4 * n + 2 * m * n + (2 * n if c["bias"] else 0), "flops": 2 * m * n * k}
    routes = c["tokens"] * c["top"]
    if c["op"] == "route":
        size = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": c["tokens"] * c["experts"] * size + 12 * routes + 4 * c["experts"] * (2 if c["bias"] else 1) + 4,
                "flops": 10 * c["tokens"] * c["experts"]}
    # the experts that routes without preference touch, on average
    touched = c["experts"] * (1 - (1 - c["top"] / c["experts"]) ** c["tokens"])
    x_rows, y_rows = (routes, c["tokens"]) if c["combine"] else (c["tokens"], routes)
    return {"bytes": int(touched * c["n"] * (c["k"] + 4)) + x_rows * (c["k"] + 4) + 2 * y_rows * c["n"] + 4 * routes
            + 4 * c["experts"] + 4 + (4 * routes if c["combine"] else 0), "flops": 2 * routes * c["n"] * c["k"]}


# ------------------------------------------------------------------- inputs

def _codes(x):
    """fp32 [..., k], values of at most 16 bits -> int8 codes, fp32 scales [...].  127 x / max|x| in 64 bits: the quotient
    of such values is never so near to a half that it is taken for one."""
    top = x.abs().amax(-1, keepdim=True)
    q = 127.0 * x.double() / torch.where(top == 0, torch.ones_like(top), top).double()
    return torch.floor(q + 0.5).to(torch.int8), (top / 127.0).squeeze(-1)


def _weights(gen, shape):
    """Codes of weights: every row reaches 127 or -127; scales that make products of unit size."""
    w = torch.randn(shape, generator=gen, device="cuda")
    w *= 127.0 / w.abs().amax(-1, keepdim=True)
    scales = shape[-1] ** -0.5 / 32 * torch.exp(0.2 * torch.randn(shape[:-1], generator=gen, device="cuda"))
    return w.round_().to(torch.int8), scales


def _rows(gen, m, k, dtype):
    """Activations in 16 bits: a few channels several times as large as the rest."""
    gain = torch.exp(0.5 * torch.randn(k, generator=gen, device="cuda"))
    return (torch.randn((m, k), generator=gen, device="cuda") * gain).to(dtype)


def _preferred(gen, tokens, experts, spread):
    """Router outputs: some experts are liked by all tokens more than others."""
    liked = spread * torch.randn(experts, generator=gen, device="cuda")
    return torch.randn((tokens, experts), generator=gen, device="cuda") + liked


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=c)
    if c["op"] == "route":
        t, e = c["tokens"], c["experts"]
        s["logits"] = (2.0 * _preferred(gen, t, e, 0.3)).to(_TYPES[c["dtype"]])
        s["bias"] = 0.05 * torch.randn(e, generator=gen, device="cuda") if c["bias"] else None
        s["chosen"] = torch.empty((t, c["top"]), dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty((t, c["top"]), device="cuda")
        s["order"] = torch.empty(t * c["top"], dtype=torch.int32, device="cuda")
        s["ends"] = torch.empty(e + 1, dtype=torch.int32, device="cuda")
        s["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        return s
    n, k, dtype = c["n"], c["k"], _TYPES[c["dtype"]]
    if c["op"] == "matmul":
        m = c["m"]
        x = _rows(gen, m, k, dtype)
        if c["step"]:
            s["x16"] = x
            s["x"] = torch.empty((m, k), dtype=torch.int8, device="cuda")
            s["x_scales"] = torch.empty(m, device="cuda")
        else:
            s["x"], s["x_scales"] = _codes(x.float())
        s["w"], s["w_scales"] = _weights(gen, (n, k))
        s["bias"] = torch.randn(n, generator=gen, device="cuda").to(dtype) if c["bias"] else None
        s["y"] = torch.empty((m, n), dtype=dtype, device="cuda")
        s["scratch"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
        return s
    t, e, top = c["tokens"], c["experts"], c["top"]
    routes = t * top
    s["x"], s["x_scales"] = _codes(_rows(gen, routes if c["combine"] else t, k, dtype).float())
    s["w"], s["w_scales"] = _weights(gen, (e, n, k))
    logits = _preferred(gen, t, e, 0.2)
    best = torch.sort(logits, dim=-1, descending=True, stable=True)
    s["chosen"] = best.indices[:, :top].to(torch.int32).contiguous()
    s["weights"] = torch.softmax(best.values[:, :top], -1).contiguous() if c["combine"] else None
    flat = s["chosen"].flatten()
    s["order"] = torch.sort(flat, dim=0, stable=True).indices.to(torch.int32)
    counts = torch.zeros(e, dtype=torch.int64, device="cuda").index_add_(0, flat.long(), torch.ones(
        routes, dtype=torch.int64, device="cuda"))
    s["ends"] = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0))).to(torch.int32)
    s["most"] = int(counts.max())
    s["y"] = torch.empty((t if c["combine"] else routes, n), dtype=dtype, device="cuda")
    s["scratch"] = torch.empty((64 << 20) + (4 * routes * n if c["combine"] else 0), dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------- the plain forms

def _plain_matmul(s):
    c = s["case"]
    x, x_scales = _codes(s["x16"].float()) if c["step"] else (s["x"], s["x_scales"])
    y = torch.matmul(x.float(), s["w"].float().t()) * x_scales[:, None] * s["w_scales"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = y.to(_TYPES[c["dtype"]])
    return {"y": y, "x_scales": x_scales} if c["step"] else {"y": y}


def _plain_route(s):
    """In 64 bits: which expert comes first depends on values that lie close to each other."""
    c = s["case"]
    t, e, g, top = c["tokens"], c["experts"], c["groups"], c["top"]
    z = s["logits"].double()
    if c["score"] == "softmax":
        p = torch.exp(z - z.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-z))
    choice = p if s["bias"] is None else p + s["bias"].double()
    ranked = torch.sort(choice.view(t, g, e // g), dim=-1, descending=True).values
    kept = torch.sort(ranked[..., :c["group_best"]].sum(-1), dim=-1, descending=True, stable=True).indices[:, :c["top_groups"]]
    inside = torch.zeros((t, g), dtype=torch.bool, device="cuda").scatter(1, kept, True)
    choice = choice.masked_fill(~inside.repeat_interleave(e // g, 1), float("-inf"))
    chosen = torch.sort(choice, dim=-1, descending=True, stable=True).indices[:, :top]
    w = p.gather(1, chosen)
    w = w / w.sum(-1, keepdim=True)
    flat = chosen.flatten()
    order = torch.sort(flat, dim=0, stable=True).indices
    ends = (flat[:, None] < torch.arange(e + 1, device="cuda")).sum(0)
    return {"chosen": chosen.to(torch.int32), "weights": w.float(), "order": order.to(torch.int32),
            "ends": ends.to(torch.int32)}


def _plain_experts(s):
    """Every expert's routes as rows of a table as long as the longest expert's."""
    c = s["case"]
    e, n, routes = c["experts"], c["n"], c["tokens"] * c["top"]
    share = routes // s["x"].shape[0]
    begin, end = s["ends"][:-1, None].long(), s["ends"][1:, None].long()
    at = begin + torch.arange(s["most"], device="cuda")
    there = at < end                                            # [experts, most]
    route = s["order"][at.clamp(max=routes - 1)].long()
    x = (s["x"][route // share].float() * there[..., None]).transpose(1, 2).contiguous()
    y = torch.bmm(s["w"].float(), x).transpose(1, 2)            # [experts, most, n]
    y = y * s["x_scales"][route // share][..., None] * s["w_scales"][:, None]
    out = torch.zeros((routes, n), device="cuda")
    out[route[there]] = y[there]
    if c["combine"]:
        out = (out.view(c["tokens"], c["top"], n) * s["weights"][..., None]).sum(1)
    return {"y": out.to(_TYPES[c["dtype"]])}


def _plain(s):
    return {"matmul": _plain_matmul, "route": _plain_route, "experts": _plain_experts}[s["case"]["op"]](s)


# ------------------------------------------------------------------ the run

def _own(s):
    import paper_2209_12982_amd as W

    c = s["case"]
    if c["op"] == "matmul":
        if c["step"]:
            W.w8_quantize(s["x16"], s["x"], s["x_scales"])
        W.w8_matmul(s["x"], s["x_scales"], s["w"], s["w_scales"], s["y"], bias=s["bias"], workspace=s["scratch"])
        return {"y": s["y"], "x_scales": s["x_scales"]} if c["step"] else {"y": s["y"]}
    if c["op"] == "route":
        W.route_experts(s["logits"], s["chosen"], s["weights"], s["order"], s["ends"], bias=s["bias"],
                        score=W.SCORE_SOFTMAX if c["score"] == "softmax" else W.SCORE_SIGMOID, groups=c["groups"],
                        top_groups=c["top_groups"], group_best=c["group_best"], workspace=s["scratch"])
        return {x: s[x] for x in ("chosen", "weights", "order", "ends")}
    W.w8_experts_matmul(s["x"], s["x_scales"], s["w"], s["w_scales"], s["order"], s["ends"], s["y"],
                        chosen=s["chosen"] if c["combine"] else None, weights=s["weights"], workspace=s["scratch"])
    return {"y": s["y"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------- the definition in 64 bits

def _quantized64(x):
    """What the codes of float64 rows stand for, and the scales."""
    scale = x.abs().amax(1) / 127
    safe = torch.where(scale > 0, scale, 1.0)[:, None]
    whole = torch.trunc(127 * x / (127 * safe))
    rest = 127 * x - whole * (127 * safe)                       # exact: both are whole multiples of a small unit
    up = (2 * rest >= 127 * safe).double()
    down = (2 * rest < -127 * safe).double()
    return (whole + up - down) * scale[:, None], scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "matmul":
        if c["step"]:
            x, scale = _quantized64(s["x16"].double())
        else:
            x, scale = s["x"].double() * s["x_scales"].double()[:, None], None
        y = x @ (s["w"].double() * s["w_scales"].double()[:, None]).t()
        if s["bias"] is not None:
            y += s["bias"].double()
        return {"y": y, "x_scales": scale} if c["step"] else {"y": y}
    if c["op"] == "route":
        if c["tokens"] * c["experts"] > 1 << 22:
            return None
        z, e = s["logits"].double().cpu(), c["experts"]
        p = torch.softmax(z, -1) if c["score"] == "softmax" else torch.sigmoid(z)
        values = (p if s["bias"] is None else p + s["bias"].double().cpu()).tolist()
        size = e // c["groups"]
        picked = []
        for row in values:
            best = [sum(sorted(row[a:a + size], reverse=True)[:c["group_best"]]) for a in range(0, e, size)]
            kept = sorted(range(c["groups"]), key=lambda i: (-best[i], i))[:c["top_groups"]]
            picked.append(sorted((i for i in range(e) if i // size in kept), key=lambda i: (-row[i], i))[:c["top"]])
        flat = [i for row in picked for i in row]
        order = sorted(range(len(flat)), key=lambda r: (flat[r], r))
        counts = [0] * (e + 1)
        for i in flat:
            counts[i + 1] += 1
        chosen = torch.tensor(picked, device="cuda")
        w = p.cuda().gather(1, chosen)
        return {"chosen": chosen.to(torch.int32), "weights": w / w.sum(1)[:, None],
                "order": torch.tensor(order, dtype=torch.int32, device="cuda"),
                "ends": torch.tensor(counts, device="cuda").cumsum(0).to(torch.int32)}
    share = c["tokens"] * c["top"] // s["x"].shape[0]
    y = torch.zeros((c["tokens"] * c["top"], c["n"]), dtype=torch.float64, device="cuda")
    flat = s["chosen"].flatten()
    for i in range(c["experts"]):
        r = (flat == i).nonzero()[:, 0]
        x = s["x"][r // share].double() * s["x_scales"][r // share, None].double()
        y[r] = x @ (s["w"][i].double() * s["w_scales"][i, :, None].double()).t()
    if c["combine"]:
        y = torch.einsum("tjn,tj->tn", y.view(c["tokens"], c["top"], -1), s["weights"].double())
    return {"y": y}

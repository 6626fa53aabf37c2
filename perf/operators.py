"""The operators of the 4-bit decoder path whose speed this framework is held
to, with the sizes and value distributions they meet in use.

A case is one call (or one step of a serving loop):

  op "matvec"  w4_matvec: a few rows times a 4-bit weight matrix
  op "append"  kv4_append: rotation and 4-bit quantization of new keys and
               values into a paged cache
  op "decode"  kv4_attention over that cache, with `step` after a kv4_append
               of the newest tokens, as a serving loop calls them
  op "prompt"  prompt_attention over packed sequences

4-bit values: 32 neighbours share a power of two 2^(s - 127), s one byte; a
code is a sign bit over the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6; two codes a
byte, the lower index in the low half.  s is the smallest with max|x| <=
6 2^(s - 127) (127 for 32 zeros), rounding goes to the nearest, ties to the
even code.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- the cases

def _matvec(name, m, n, k, dtype, bias=False):
    c = dict(op="matvec", m=m, n=n, k=k, dtype=dtype, bias=bias)
    return dict(name=name, **c) if name else c


def _append(name, seqs, tokens, heads, kv_heads, dim, rot, pairs, page, dtype):
    c = dict(op="append", seqs=seqs, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, pairs=pairs,
             page=page, dtype=dtype)
    return dict(name=name, **c) if name else c


def _decode(name, batch, q_len, longest, heads, kv_heads, dim, page, dtype, step=False):
    c = dict(op="decode", batch=batch, q_len=q_len, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim,
             page=page, dtype=dtype, step=step)
    return dict(name=name, **c) if name else c


def _prompt(name, seqs, longest, prefix, heads, kv_heads, dim, dtype):
    c = dict(op="prompt", seqs=seqs, longest=longest, prefix=prefix, heads=heads, kv_heads=kv_heads, dim=dim,
             dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token through a small projection: the smallest call, all latency
        _matvec("matvec_small", 1, 1024, 1024, "bf16"),
        # one token through a feed-forward layer's wide projection
        _matvec("matvec_token", 1, 16384, 4096, "bf16"),
        # sixteen sequences through the projection back, long sums
        _matvec("matvec_batch", 16, 4096, 16384, "fp16"),
        # odd row count (a vocabulary slice), a few rows, bias
        _matvec("matvec_odd_bias", 5, 5003, 2080, "bf16", bias=True),
        # one new token for each of 32 sequences
        _append("append_token", 32, 32, 32, 8, 128, 128, False, 16, "bf16"),
        # whole prompts entering the cache at once, half of each head rotated
        _append("append_prompt", 7, 8200, 32, 8, 128, 64, True, 64, "fp16"),
        # one short sequence, small heads: latency
        _decode("decode_one", 1, 1, 777, 8, 2, 64, 16, "fp16"),
        # a serving batch of unequal lengths, the newest token appended first
        _decode("decode_batch", 64, 1, 4096, 32, 8, 128, 64, "bf16", step=True),
        # two very long sequences: the axis has to be split
        _decode("decode_long", 2, 1, 131072, 32, 8, 128, 64, "bf16"),
        # one short prompt, small heads: latency
        _prompt("prompt_short", 1, 333, 0, 8, 2, 64, "fp16"),
        # a batch of prompts of unequal lengths, packed
        _prompt("prompt_packed", 12, 2048, 0, 32, 8, 128, "bf16"),
        # one long prompt: the matrix products bound it
        _prompt("prompt_long", 1, 16384, 0, 16, 4, 128, "bf16"),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 64 rows and 256 to 32768 outputs, 1 to
    8200 new tokens, caches of 1 to 131072 tokens a sequence, prompts of 1 to
    8192, heads of 64 to 256 in groups of 1 to 16, either type."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def heads():
        kv = rng.choice([1, 2, 3, 4, 5, 8, 16])
        return kv * rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), kv

    op = rng.choice(["matvec", "append", "decode", "decode", "prompt", "prompt"])
    while True:
        dtype = rng.choice(["bf16", "fp16"])
        hq, hkv = heads()
        dim = rng.choice([64, 96, 128, 128, 192, 256])
        page = rng.choice([16, 32, 64, 128])
        if op == "matvec":
            c = _matvec(None, log_int(1, 64), log_int(256, 32768), 32 * log_int(8, 512), dtype, rng.random() < 0.3)
            small = c["n"] * c["k"] <= 1 << 27
        elif op == "append":
            t = log_int(1, 8200)
            rot = rng.choice([dim, dim, dim // 2])
            c = _append(None, min(t, log_int(1, 64)), t, hq, hkv, dim, rot, rng.random() < 0.5, page, dtype)
            small = hq <= 64 and t * (hq + 2 * hkv) * dim <= 8200 * 48 * 128
        elif op == "decode":
            c = _decode(None, log_int(1, 128), rng.choice([1, 1, 1, 1, 2, 4, 5, 8]), log_int(1, 131072), hq, hkv, dim,
                        page, dtype, rng.random() < 0.5)
            small = hq <= 64 and c["batch"] * c["longest"] * hkv * dim <= 2 * 131072 * 8 * 128
            small = small and c["batch"] * c["longest"] * c["q_len"] * hq <= 2 * 131072 * 64
        else:
            c = _prompt(None, log_int(1, 16), log_int(1, 8192), rng.choice([0, 0, 0, 100, 1000]), hq, hkv, dim, dtype)
            t = c["longest"] + c["prefix"]
            small = hq <= 64 and c["seqs"] * c["longest"] * t * hq * max(dim, 128) <= 16384 * 16384 * 16 * 64
        if small and not any(v == 3072 for v in c.values()):
            return c


def _fixed(case, *more):
    """A generator that depends on the case's sizes alone."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")) + repr(more))


def _lengths(case, count, longest):
    """`count` lengths from 1 to `longest`, evenly spread over the logarithm's upper part, the first the longest; one
    in a dozen is empty."""
    rng = _fixed(case, "lengths")
    got = [longest]
    for _ in range(count - 1):
        got.append(0 if rng.random() < 1 / 12 else max(1, int(longest * math.exp(rng.uniform(-3.0, 0.0)))))
    return got


def _split(case, total, count):
    """`total` tokens dealt out to `count` sequences, one at least to each."""
    rng = _fixed(case, "split")
    cuts = sorted(rng.sample(range(1, total), count - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _visible(q_len, k_len):
    """Pairs that a causal mask aligned to the end of the keys leaves."""
    first = k_len - q_len + 1                       # keys that the first query sees
    if first >= 1:
        return q_len * first + q_len * (q_len - 1) // 2
    return k_len * (k_len + 1) // 2


def work(case):
    c = case
    if c["op"] == "matvec":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": n * k // 2 + n * k // 32 + 2 * m * k + 2 * m * n + (2 * n if c["bias"] else 0),
                "flops": 2 * m * n * k}
    d, hq, hkv = c["dim"], c["heads"], c["kv_heads"]
    token = hkv * (d + d // 16)                     # bytes of one token's keys and values in the cache
    if c["op"] == "append":
        t = c["tokens"]
        return {"bytes": 4 * t * (hq + 2 * hkv) * d + t * token + t * (4 * c["rot"] + 12),
                "flops": 3 * t * (hq + hkv) * c["rot"] + 4 * t * 2 * hkv * d}
    if c["op"] == "decode":
        lens = _lengths(c, c["batch"], c["longest"])
        rows = c["batch"] * c["q_len"]
        pairs = sum(_visible(c["q_len"], n) for n in lens)
        b = sum(lens) * token + 4 * rows * hq * d
        if c["step"]:
            b += 4 * rows * (hq + 2 * hkv) * d
        return {"bytes": b, "flops": 4 * pairs * hq * d}
    q_lens = _lengths(c, c["seqs"], c["longest"])
    keys = [n + c["prefix"] for n in q_lens]
    pairs = sum(_visible(q, k) for q, k in zip(q_lens, keys))
    return {"bytes": 4 * sum(q_lens) * hq * d + 4 * sum(keys) * hkv * d, "flops": 4 * pairs * hq * d}


# ---------------------------------------------------- 4-bit values in torch

_MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _encode(x):
    """fp32 [..., d] -> codes uint8 [..., d/2] and scales uint8 [..., d/32]."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    mant, ex = torch.frexp(g.abs().amax(-1))
    e = ex - torch.where(mant <= 0.75, 3, 2)
    e = torch.where(mant == 0, torch.zeros_like(e), e).clamp(-127, 127)
    a = torch.ldexp(g, -e.unsqueeze(-1))
    s = torch.signbit(g)
    a = a.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * s).to(torch.uint8).reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode4(codes, scales):
    """The fp32 values of codes uint8 [..., d/2] with scales uint8 [..., d/32]."""
    table = torch.tensor(_MAGNITUDES + [-v for v in _MAGNITUDES], device=codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    g = v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32)
    return torch.ldexp(g, (scales.int() - 127).unsqueeze(-1)).reshape(v.shape)


def _rotate(x, cos, sin, pairs):
    """fp32 [t, heads, d]; cos, sin [t, r/2]: the first r dims turned, as halves or as neighbours."""
    h = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if pairs else (x[..., :h], x[..., h:2 * h])
    u, w = a * c - b * s, b * c + a * s
    y = torch.stack((u, w), -1).flatten(-2) if pairs else torch.cat((u, w), -1)
    return torch.cat((y, x[..., 2 * h:]), -1)


# ------------------------------------------------------------------- inputs

def _table(case, positions):
    r = case.get("rot", case["dim"])
    f = 10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.cat((a.cos(), a.sin()), -1).float()


def _keys(gen, shape, dtype):
    """Keys and values: a few channels several times as large as the rest."""
    d = shape[-1]
    gain = torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda"))
    return (torch.randn(shape, generator=gen, device="cuda") * gain).to(dtype)


def _empty_cache(pages, hkv, page, d):
    return tuple(torch.zeros((pages, hkv, page, w), dtype=torch.uint8, device="cuda")
                 for w in (d // 2, d // 32, d // 2, d // 32))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES[c["dtype"]]
    s = dict(case=c)
    if c["op"] == "matvec":
        m, n, k = c["m"], c["n"], c["k"]
        s["x"] = torch.randn((m, k), generator=gen, device="cuda").to(dtype)
        w = torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5
        s["codes"], s["scales"] = _encode(w)
        s["bias"] = torch.randn(n, generator=gen, device="cuda").to(dtype) if c["bias"] else None
        s["y"] = torch.empty((m, n), dtype=dtype, device="cuda")
        s["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        return s
    d, hq, hkv = c["dim"], c["heads"], c["kv_heads"]
    s["scale"] = d ** -0.5
    if c["op"] == "prompt":
        q_lens = _lengths(c, c["seqs"], c["longest"])
        k_lens = [n + c["prefix"] for n in q_lens]
        s["q"] = torch.randn((sum(q_lens), hq, d), generator=gen, device="cuda").to(dtype)
        s["k"] = _keys(gen, (sum(k_lens), hkv, d), dtype)
        s["v"] = _keys(gen, (sum(k_lens), hkv, d), dtype)
        s["cu_q"] = torch.tensor([0] + q_lens, device="cuda").cumsum(0).to(torch.int32)
        s["cu_k"] = torch.tensor([0] + k_lens, device="cuda").cumsum(0).to(torch.int32)
        s["longest_q"], s["longest_k"] = max(q_lens), max(k_lens)
        s["out"] = torch.empty_like(s["q"])
        return s
    page = c["page"]
    if c["op"] == "append":
        lens = _split(c, c["tokens"], c["seqs"])
        held = 64 if c["tokens"] == c["seqs"] else 0        # single tokens join sequences that are there already
        counts = [-(-(n + held) // page) for n in lens]
        t = c["tokens"]
    else:
        lens = _lengths(c, c["batch"], c["longest"])
        counts = [-(-n // page) for n in lens]
        t = c["batch"] * c["q_len"]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=gen, device="cuda")
    rows = torch.full((len(lens), max(max(counts), 1)), -1, dtype=torch.int64)
    at = 0
    order_host = order.cpu()
    for i, n in enumerate(counts):
        rows[i, :n] = order_host[at:at + n]
        at += n
    table = rows.cuda()
    seq, pos = [], []
    if c["op"] == "append":
        for i, n in enumerate(lens):
            seq += [i] * n
            pos += list(range(held, held + n))
    else:
        for i, n in enumerate(lens):                        # the newest q_len tokens of each sequence
            seq += [i] * c["q_len"]
            pos += list(range(n - c["q_len"], n))
    seq, pos = torch.tensor(seq, device="cuda"), torch.tensor(pos, device="cuda")
    there = pos >= 0                                        # a sequence shorter than q_len: its first rows are padding
    pos = pos.clamp(min=0)
    slots = table[seq, pos // page] * page + pos % page
    s["slots"] = torch.where(there, slots, torch.full_like(slots, -1))
    s["positions"] = pos.to(torch.int32)
    s["cos_sin"] = _table(c, max(1, int(pos.max()) + 1))
    qkv = torch.randn((t, hq + 2 * hkv, d), generator=gen, device="cuda")
    s["q"], k, v = qkv.to(dtype).split((hq, hkv, hkv), 1)   # slices of one projection's output, as they come
    s["k"] = k * torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda")).to(dtype)
    s["v"] = v
    s["q_out"] = torch.empty((t, hq, d), dtype=dtype, device="cuda")
    s["k_out"] = torch.empty((t, hkv, d), dtype=dtype, device="cuda")
    s["v_out"] = torch.empty((t, hkv, d), dtype=dtype, device="cuda")
    if c["op"] == "append":
        s["cache"] = _empty_cache(pages, hkv, page, d)
        return s
    kc, ks = _encode(_keys(gen, (pages, hkv, page, d), torch.float32))
    vc, vs = _encode(_keys(gen, (pages, hkv, page, d), torch.float32))
    s["cache"] = (kc, ks, vc, vs)
    s["block_table"] = table.to(torch.int32)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q_rows"] = s["q"].contiguous()
    s["out"] = torch.empty((t, hq, d), dtype=dtype, device="cuda")
    s["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------- the plain forms

def _plain_append(s):
    c = s["case"]
    dtype, page = _TYPES[c["dtype"]], c["page"]
    cos, sin = s["cos_sin"][s["positions"].long()].chunk(2, -1)
    q = _rotate(s["q"].float(), cos, sin, c.get("pairs", False))
    k = _rotate(s["k"].float(), cos, sin, c.get("pairs", False))
    kc, ks = _encode(k)
    vc, vs = _encode(s["v"].float())
    there = (s["slots"] >= 0).nonzero().squeeze(1)
    p, o = s["slots"][there] // page, s["slots"][there] % page
    for held, new in zip(s["cache"], (kc, ks, vc, vs)):
        held[p, :, o] = new[there]
    return q.to(dtype), _decode4(kc, ks).to(dtype), _decode4(vc, vs).to(dtype)


def _softmax_product(scores, seen, v):
    """softmax over the last axis where `seen`, times v; 0 for a row that sees nothing."""
    scores = scores.masked_fill(~seen, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_decode(s, q):
    c = s["case"]
    b, ql, hq, hkv, d, page = c["batch"], c["q_len"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    t = s["block_table"].clamp(min=0).long()

    def whole(codes, scales):                               # [b, hkv, tokens, d]
        x = _decode4(codes[t], scales[t])                   # [b, pages, hkv, page, d]
        return x.transpose(1, 2).reshape(b, hkv, -1, d)

    k, v = whole(*s["cache"][:2]), whole(*s["cache"][2:])
    n = k.shape[2]
    rows = q.float().view(b, ql, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    scores = torch.matmul(rows, k.transpose(2, 3)) * s["scale"]
    last = s["lens"][:, None] - ql + torch.arange(ql, device="cuda")
    seen = torch.arange(n, device="cuda") <= last[..., None]                    # [b, ql, n]
    seen = seen[:, None, None].expand(b, 1, hq // hkv, ql, n).reshape(b, 1, -1, n)
    o = _softmax_product(scores, seen, v)
    o = o.view(b, hkv, hq // hkv, ql, d).permute(0, 3, 1, 2, 4).reshape(b * ql, hq, d)
    return o.to(_TYPES[c["dtype"]])


def _padded(x, cu, longest):
    """Packed [total, heads, d] -> fp32 [seqs, heads, longest, d], zeros after each sequence's end."""
    at = cu[:-1, None].long() + torch.arange(longest, device="cuda")
    there = at < cu[1:, None]
    y = x[at.clamp(max=max(x.shape[0] - 1, 0))].float() * there[..., None, None]
    return y.transpose(1, 2).contiguous(), at, there


def _plain_prompt(s):
    c = s["case"]
    hq, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    q, at, there = _padded(s["q"], s["cu_q"], s["longest_q"])
    k, _, _ = _padded(s["k"], s["cu_k"], s["longest_k"])
    v, _, _ = _padded(s["v"], s["cu_k"], s["longest_k"])
    n, g = q.shape[0], hq // hkv
    q = q.view(n, hkv, g * s["longest_q"], d)
    scores = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    q_len, k_len = s["cu_q"].diff(), s["cu_k"].diff()
    i, j = torch.arange(s["longest_q"], device="cuda"), torch.arange(s["longest_k"], device="cuda")
    last = (k_len - q_len)[:, None] + i
    seen = (j <= last[..., None]) & (j < k_len[:, None, None])                  # [n, q, k]
    seen = seen[:, None, None].expand(n, 1, g, len(i), len(j)).reshape(n, 1, -1, len(j))
    o = _softmax_product(scores, seen, v).view(n, hq, len(i), d).transpose(1, 2)
    out = torch.zeros(s["q"].shape, device="cuda")
    out[at[there]] = o[there]
    return out.to(_TYPES[c["dtype"]])


def _plain(s):
    c = s["case"]
    if c["op"] == "matvec":
        y = torch.matmul(s["x"].float(), _decode4(s["codes"], s["scales"]).t())
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return {"y": y.to(_TYPES[c["dtype"]])}
    if c["op"] == "append":
        q, k, v = _plain_append(s)
        return {"q": q, "k": k, "v": v}
    if c["op"] == "decode":
        if not c["step"]:
            return {"o": _plain_decode(s, s["q_rows"])}
        q, k, v = _plain_append(s)
        return {"o": _plain_decode(s, q), "k": k, "v": v}
    return {"o": _plain_prompt(s)}


# ------------------------------------------------------------------ the run

def _own(s):
    import paper_2209_12982_amd as W

    c = s["case"]
    if c["op"] == "matvec":
        W.w4_matvec(s["x"], s["codes"], s["scales"], s["y"], bias=s["bias"], workspace=s["scratch"])
        return {"y": s["y"]}
    if c["op"] == "prompt":
        W.prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["longest_q"], s["out"], s["scale"])
        return {"o": s["out"]}
    q, got = s.get("q_rows"), {}
    if c["op"] == "append" or c["step"]:
        W.kv4_append(s["q"], s["k"], s["v"], s["cos_sin"], s["positions"], s["slots"], s["cache"], s["q_out"],
                     s["k_out"], s["v_out"], rotary=W.ROTARY_PAIRS if c.get("pairs") else W.ROTARY_HALVES,
                     values=W.KV4_CACHED)
        q, got = s["q_out"], {"k": s["k_out"], "v": s["v_out"]}
        if c["op"] == "append":
            return {"q": q, **got}
    W.kv4_attention(q, s["cache"], s["block_table"], s["lens"], s["out"], s["scale"], workspace=s["scratch"])
    return {"o": s["out"], **got}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------- the definition in 64 bits

def _value64(codes, scales):
    """Codes and scales by their bits: sign, two exponent bits, one mantissa bit."""
    both = torch.stack((codes % 16, codes // 16), -1).flatten(-2).to(torch.float64)
    sign = 1.0 - 2.0 * (both >= 8).double()
    mag = both % 8
    ex, man = torch.floor(mag / 2), mag % 2
    v = torch.where(ex == 0, man / 2, (1 + man / 2) * 2.0 ** (ex - 1)) * sign
    return v * (2.0 ** (scales.double() - 127)).repeat_interleave(32, -1)


def _nearest64(x):
    """The 4-bit values nearest to float64 x, in groups of 32 along the last axis."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 6))
    e = torch.where(top > 6 * 2.0 ** e, e + 1, e)
    e = torch.where(top <= 6 * 2.0 ** (e - 1), e - 1, e)
    e = torch.where(top == 0, torch.zeros_like(e), e).clamp(-127, 127)
    a = g.abs() * 2.0 ** -e
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.round(a / step) * step * torch.sign(g) * 2.0 ** e).flatten(-2)


def _turn64(x, cos, sin, pairs):
    h = cos.shape[-1]
    y = x.clone()
    i = torch.arange(h, device=x.device)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + h)
    z = torch.complex(x[..., a], x[..., b]) * torch.complex(cos, sin)[:, None]
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _attend64(q, k, v, first, scale):
    """q [n, d], k, v [t, d]: row i sees the keys up to index first[i]."""
    out = torch.zeros_like(q)
    for a in range(0, q.shape[0], 2048):
        z = (q[a:a + 2048] @ k.t()) * scale
        z.masked_fill_(torch.arange(k.shape[0], device=q.device) > first[a:a + 2048, None], float("-inf"))
        some = first[a:a + 2048] >= 0
        out[a:a + 2048][some] = torch.softmax(z[some], -1) @ v
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "matvec":
        y = s["x"].double() @ _value64(s["codes"], s["scales"]).t()
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    hq, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    g = hq // hkv
    if c["op"] == "prompt":
        o = torch.zeros((s["q"].shape[0], hq, d), dtype=torch.float64, device="cuda")
        cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
        for i in range(c["seqs"]):
            n, t = cq[i + 1] - cq[i], ck[i + 1] - ck[i]
            if not n or not t:
                continue
            for h in range(hq):
                k, v = (s[x][ck[i]:ck[i + 1], h // g].double() for x in "kv")
                o[cq[i]:cq[i + 1], h] = _attend64(s["q"][cq[i]:cq[i + 1], h].double(), k, v,
                                                  torch.arange(t - n, t, device="cuda"), s["scale"])
        return {"o": o}
    got = {}
    if c["op"] == "append" or c["step"]:
        cos, sin = s["cos_sin"].double()[s["positions"].long()].chunk(2, -1)
        q = _turn64(s["q"].double(), cos, sin, c.get("pairs", False))
        k = _nearest64(_turn64(s["k"].double(), cos, sin, c.get("pairs", False)))
        v = _nearest64(s["v"].double())
        got = {"k": k, "v": v}
        if c["op"] == "append":
            return {"q": q, **got}
    else:
        q = s["q_rows"].double()
    ql, page = c["q_len"], c["page"]
    o = torch.zeros((c["batch"] * ql, hq, d), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        if not n:
            continue
        pages = s["block_table"][b, :-(-n // page)].long()
        kk, vv = (_value64(s["cache"][i][pages], s["cache"][i + 1][pages]).transpose(0, 1).flatten(1, 2)[:, :n]
                  for i in (0, 2))
        if c["step"]:
            new = min(ql, n)
            rows = slice((b + 1) * ql - new, (b + 1) * ql)
            kk, vv = kk.clone(), vv.clone()
            kk[:, n - new:], vv[:, n - new:] = got["k"][rows].transpose(0, 1), got["v"][rows].transpose(0, 1)
        first = torch.arange(n - ql, n, device="cuda")
        # the kernel's own rounding of the turned queries is part of the step: they are an output of its first call
        qb = q[b * ql:(b + 1) * ql]
        if c["step"]:
            qb = qb.to(_TYPES[c["dtype"]]).double()
        for h in range(hq):
            o[b * ql:(b + 1) * ql, h] = _attend64(qb[:, h], kk[h // g], vv[h // g], first, s["scale"])
    return {"o": o, **got}

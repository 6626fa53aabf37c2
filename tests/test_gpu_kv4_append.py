"""kv4_append: codes and scales exactly as the oracle has them (its rotation
rounds as the operator's definition says, so there is one right answer), the
outputs exactly too, and the rest of the cache untouched.  The rotation itself
is held against float64: three roundings of values up to |u| + |w|, then one to
the 16-bit type."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder

from decoder_util import ROUND, TINY, dtype, half, host
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def _cache(torch, pages, hkv, page, d, fill=0xA5):
    return tuple(torch.full((pages, hkv, page, w), fill, dtype=torch.uint8, device="cuda")
                 for w in (d // 2, d // 32, d // 2, d // 32))


def _angles(rng, rows, rot):
    a = rng.uniform(-4, 4, (rows, rot // 2))
    return np.concatenate((np.cos(a), np.sin(a)), -1).astype(np.float32)


def _run(torch, rng, tokens, hq, hkv, d, rot, pairs, page, name, values, k_edit=None):
    """Calls the operator on the slices of one projection's output and compares
    everything with the oracle; returns the cache."""
    pages = tokens // page + 3
    big = np.concatenate([rng.normal(0, 1, (tokens, hq, d)),
                          rng.normal(0, 1, (tokens, hkv, d)) * np.exp(rng.normal(0, 2, (tokens, hkv, d))),
                          rng.normal(0, 1, (tokens, hkv, d)) * np.exp2(rng.integers(-9, 5, (tokens, 1, 1)))], 1)
    if k_edit:
        k_edit(big[:, hq:hq + hkv])
    x, xv = half(torch, big, name)
    q, k, v = x.split((hq, hkv, hkv), 1)
    cs = _angles(rng, 50, rot)
    pos = rng.integers(0, 50, tokens).astype(np.int32)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 3:
        slots[1], slots[tokens - 1], pos[2] = -1, pages * page + 5, 50
    if tokens > 5:
        slots[3], pos[4] = np.int64(1) << 62, -7
    dt = dtype(torch, name)
    cache = _cache(torch, pages, hkv, page, d)
    outs = [torch.full((tokens, h, d), 3.0, dtype=dt, device="cuda") for h in (hq, hkv, hkv)]
    W.kv4_append(q if hq else None, k, v, torch.from_numpy(cs).cuda(), torch.from_numpy(pos).cuda(),
                 torch.from_numpy(slots).cuda(), cache, outs[0] if hq else None, outs[1], outs[2],
                 rotary=W.ROTARY_PAIRS if pairs else W.ROTARY_HALVES, values=values)
    torch.cuda.synchronize()

    placed = (pos >= 0) & (pos < 50)
    rows = cs[np.where(placed, pos, 0)]
    x32 = xv.astype(np.float32)
    turned_q = decoder.rotate(x32[:, :hq], rows, pairs)
    turned_k = decoder.rotate(x32[:, hq:hq + hkv], rows, pairs)
    vals = x32[:, hq + hkv:]
    kc, ks = decoder.encode(turned_k)
    vc, vs = decoder.encode(vals)
    want = [np.full((pages, hkv, page, c.shape[-1]), 0xA5, np.uint8) for c in (kc, ks, vc, vs)]
    for t in range(tokens):
        if placed[t] and 0 <= slots[t] < pages * page:
            for w, new in zip(want, (kc, ks, vc, vs)):
                w[slots[t] // page, :, slots[t] % page] = new[t]
    for w, got, what in zip(want, cache, ("k_codes", "k_scales", "v_codes", "v_scales")):
        g = got.cpu().numpy()
        assert (g == w).all(), f"{what}: {(g != w).sum()} of {g.size} bytes differ"

    def same(got, ref, what):
        r = torch.from_numpy(np.ascontiguousarray(ref)).to(dt)
        r[torch.from_numpy(~placed)] = float("nan")
        a, b = got.cpu().view(torch.int16), r.view(torch.int16)
        differ = (a != b) & ~(torch.isnan(got.cpu()) & torch.isnan(r)) & ~((got.cpu() == 0) & (r == 0))
        assert not differ.any(), f"{what}: {int(differ.sum())} of {differ.numel()} differ"

    if hq:
        same(outs[0], turned_q, "q_out")
        # the rotation against float64
        h = rot // 2
        j = np.arange(h)
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + h)
        z = (xv[:, :hq][..., a] + 1j * xv[:, :hq][..., b]) * (rows[:, None, :h].astype(float) + 1j * rows[:, None, h:])
        ref = xv[:, :hq].copy()
        ref[..., a], ref[..., b] = z.real, z.imag
        size = xv[:, :hq].__abs__().copy()
        size[..., a] = size[..., b] = np.abs(xv[:, :hq][..., a]) + np.abs(xv[:, :hq][..., b])
        err = 3 * 2.0 ** -24 * size
        bound = err + ROUND[name] * (np.abs(ref) + err) + TINY[name]
        assert (np.abs(host(outs[0]) - ref) <= bound)[placed].all()
    same(outs[1], decoder.decode(kc, ks) if values == W.KV4_CACHED else turned_k, "k_out")
    same(outs[2], decoder.decode(vc, vs) if values == W.KV4_CACHED else vals, "v_out")
    return cache


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("tokens,hq,hkv,d,rot,page", [
    (1, 1, 1, 64, 64, 16), (7, 4, 2, 128, 128, 16), (33, 3, 3, 96, 96, 48), (18, 8, 1, 128, 64, 64),
    (5, 2, 1, 256, 256, 32), (9, 6, 2, 192, 96, 16), (11, 2, 2, 128, 0, 16), (6, 0, 2, 64, 32, 16),
    (4, 2, 1, 32, 16, 16), (130, 5, 5, 64, 16, 128)])
def test_append(tokens, hq, hkv, d, rot, page, pairs, name):
    torch = torch_dev()
    rng = np.random.default_rng(tokens + 10 * hq + 100 * d + rot)
    _run(torch, rng, tokens, hq, hkv, d, rot, pairs, page, name, W.KV4_CACHED if tokens % 2 else W.KV4_ROTATED)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
def test_append_ties_zeros_and_not_finite(name):
    """No rotation, so the keys reach the quantizer as they are: every tie between
    two codes, a group of zeros of either sign, the largest and smallest
    magnitudes, groups with an infinity or a NaN beside sound ones."""
    torch = torch_dev()

    def edit(k):
        ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
        k[0, 0, :32] = np.tile(np.concatenate([ties, -ties]), 2) * 2.0 ** -3
        k[0, 0, 32:64] = 0.0
        k[0, 0, 40] = -0.0
        k[1, 0, :32] = 2.0 ** -24 * np.arange(32)          # fp16's subnormals
        k[2, 0, :32] = 65504.0
        k[3, 0, 5] = np.inf
        k[4, 0, 37] = np.nan
        k[5, 0, :32] = 6.0 * 2.0 ** -2                      # a maximum exactly at 6 * 2^e
        k[5, 0, 0] = -6.0 * 2.0 ** -2

    for values in (W.KV4_ROTATED,):
        _run(torch, np.random.default_rng(8), 8, 2, 2, 64, 0, False, 16, name, values, edit)


def test_append_extreme_exponents():
    """bf16 reaches scales that a byte barely holds: 2^-133 .. 2^127."""
    torch = torch_dev()

    def edit(k):
        k[0, 0, :32] = 2.0 ** -133 * (1 + np.arange(32) % 3)
        k[0, 0, 32:64] = 2.0 ** -126
        k[3, 0, :32] = 3.0e38
        k[5, 0, :32] = 2.0 ** np.arange(-16, 16) * 2.0 ** 100

    _run(torch, np.random.default_rng(9), 8, 2, 1, 64, 0, False, 16, "bf16", W.KV4_CACHED, edit)


def test_append_without_outputs_and_without_cache():
    torch = torch_dev()
    rng = np.random.default_rng(10)
    k, _ = half(torch, rng.normal(0, 1, (3, 2, 64)), "bf16")
    cs = torch.from_numpy(_angles(rng, 9, 64)).cuda()
    pos = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    slots = torch.tensor([4, 5, 6], device="cuda")
    cache = _cache(torch, 2, 2, 16, 64)
    W.kv4_append(None, k, k, cs, pos, slots, cache)
    assert int((cache[0] != 0xA5).sum()) > 0
    out = torch.zeros_like(k)
    W.kv4_append(None, k, k, cs, pos, slots, _cache(torch, 0, 2, 16, 64), v_out=out)      # no pages: all padding
    assert (out == k).all()
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    W.kv4_append(None, none, none, cs, pos[:0], slots[:0], cache)


def test_append_past_four_gigabytes():
    """Slots whose bytes lie beyond 2^32 of the cache's start."""
    torch = torch_dev()
    d, hkv, page = 256, 8, 128
    pages = (9 << 29) // (hkv * page * d // 2)
    cache = (torch.empty((pages, hkv, page, d // 2), dtype=torch.uint8, device="cuda"),
             torch.empty((pages, hkv, page, d // 32), dtype=torch.uint8, device="cuda"))
    cache = cache + tuple(torch.empty_like(c) for c in cache)
    assert cache[0].numel() > 1 << 32
    rng = np.random.default_rng(11)
    k, kv = half(torch, rng.normal(0, 1, (2, hkv, d)), "fp16")
    slots = torch.tensor([pages * page - 1, pages * page // 2 + 77], device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    W.kv4_append(None, k, k, torch.zeros((1, 0), device="cuda"), pos, slots, cache)
    kc, ks = decoder.encode(kv.astype(np.float32))
    for t, s in enumerate(slots.tolist()):
        assert (cache[0][s // page, :, s % page].cpu().numpy() == kc[t]).all()
        assert (cache[3][s // page, :, s % page].cpu().numpy() == ks[t]).all()


def test_append_refuses_other_tensors():
    torch = torch_dev()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    q, k, cs = z(4, 4, 64), z(4, 2, 64), z(9, 64, dt=torch.float32)
    pos, slots = z(4, dt=torch.int32), z(4, dt=torch.int64)
    cache = _cache(torch, 2, 2, 16, 64)
    for bad in (lambda: W.kv4_append(q, k, k, cs, pos, slots, cache),                       # queries without q_out
                lambda: W.kv4_append(q.half(), k, k, cs, pos, slots, cache, q),
                lambda: W.kv4_append(None, k, k[:, :1], cs, pos, slots, cache),
                lambda: W.kv4_append(None, k, k, cs.double(), pos, slots, cache),
                lambda: W.kv4_append(None, k, k, cs, pos.long(), slots, cache),
                lambda: W.kv4_append(None, k, k, cs, pos, slots[:3], cache),
                lambda: W.kv4_append(None, k, k, cs, pos, slots, cache[:3] + (cache[3][:1],)),
                lambda: W.kv4_append(None, k[:, :1], k[:, :1], cs, pos, slots, cache),
                lambda: W.kv4_append(None, k.cpu(), k, cs, pos, slots, cache)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: W.kv4_append(None, k, k, z(9, 80, dt=torch.float32), pos, slots, cache), -1),
                        (lambda: W.kv4_append(None, k, k, z(9, 24, dt=torch.float32), pos, slots, cache), -2),
                        (lambda: W.kv4_append(None, k, k, cs, pos, slots, cache, rotary=2), -1),
                        (lambda: W.kv4_append(None, k, k, cs, pos, slots, _cache(torch, 2, 2, 24, 64)), -2)):
        with pytest.raises(W.WinoError) as e:
            bad()
        assert e.value.status == status


def test_append_no_tokens_with_queries():
    torch = torch_dev()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    cache = _cache(torch, 2, 2, 16, 64)
    W.kv4_append(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), z(9, 64, dt=torch.float32), z(0, dt=torch.int32),
                 z(0, dt=torch.int64), cache, z(0, 4, 64), z(0, 2, 64), z(0, 2, 64))
    assert all(bool((c == 0xA5).all()) for c in cache)


def test_append_cached_values_that_fp16_rounds():
    """The cache holds 65536 for keys of 60000 and exact values under small scales; k_out has them rounded to fp16,
    infinity for the former."""
    torch = torch_dev()
    d, tokens = 64, 2
    cs = np.concatenate((np.full((1, 16), 2.0 ** -5), np.zeros((1, 16))), -1).astype(np.float32)     # "cosines" that scale
    k = np.zeros((tokens, 1, d), np.float32)
    k[0, 0, :], k[0, 0, 40] = 60000.0, -65504.0
    k[1, 0, :32] = 2.0 ** -24 * (1 + np.arange(32) % 3)
    kt, kv = half(torch, k, "fp16")
    cache, out = _cache(torch, 1, 1, 16, d, 0), torch.zeros_like(kt)
    i = lambda t: torch.zeros(tokens, dtype=t, device="cuda")  # noqa: E731
    W.kv4_append(None, kt, kt, torch.from_numpy(cs).cuda(), i(torch.int32), torch.arange(tokens, device="cuda"), cache,
                 k_out=out, values=W.KV4_CACHED)
    held = decoder.decode(cache[0].cpu().numpy()[0, 0, :tokens], cache[1].cpu().numpy()[0, 0, :tokens])
    assert (held[0, 32:] == np.where(np.arange(32, 64) == 40, -65536.0, 65536.0)).all()
    assert np.isinf(host(out)[0, 0, 32:]).all()
    assert (held[1, :32] == kv[1, 0, :32] * 2.0 ** -5).all() and (held[1, :32] > 0).all()
    assert (host(out)[:, 0] == torch.from_numpy(held).to(torch.float16).double().numpy()).all()
    assert (host(out)[1, 0, :32] == 0).all()

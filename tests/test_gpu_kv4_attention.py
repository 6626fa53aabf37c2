"""kv4_attention against softmax attention in float64 over the same 4-bit
cache.  Element-wise bound: decoder_util.attention_bound, with probabilities
held to 2^-16 (they may be split in two bf16 numbers for the matrix cores)."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder

from decoder_util import attention_bound, dtype, half, host, paged
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu

EPS_P = 2.0 ** -16


def _setup(torch, rng, lens, q_len, hq, hkv, d, page, name, gain=1.0):
    table, pages = paged(rng, lens, page)
    shape = (pages, hkv, page)
    kc, vc = (rng.integers(0, 256, shape + (d // 2,), dtype=np.uint8) for _ in range(2))
    ks, vs = (rng.integers(124, 129, shape + (d // 32,), dtype=np.uint8) for _ in range(2))
    used = np.zeros((pages, page), bool)
    for b, n in enumerate(lens):
        for t in range(n):
            used[table[b, t // page], t % page] = True
    for s in (ks, vs):                                   # nothing has been written there: scales that read as NaN
        s.transpose(0, 2, 1, 3)[~used] = 255
    q, qv = half(torch, gain * rng.normal(0, 1, (len(lens) * q_len, hq, d)), name)
    return table, (kc, ks, vc, vs), q, qv


def _call(torch, q, cache, table, lens, scale, workspace=None, stream=None):
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    W.kv4_attention(q, tuple(torch.from_numpy(c).cuda() for c in cache), torch.from_numpy(table).cuda(),
                    torch.tensor(lens, dtype=torch.int32, device="cuda"), out, scale, workspace=workspace, stream=stream)
    return out


def _workspace(torch, lens, q_len, hq, hkv, d, table, page):
    n = W.kv4_attention_workspace_bytes(len(lens), q_len, hq, hkv, d, table.shape[1], page)
    return torch.full((n + 16,), 255, dtype=torch.uint8, device="cuda")


def _reference(cache, table, lens, qv, q_len, hq, hkv, d, page, scale, name, hidden=()):
    """(result, bound) for every row; `hidden`: tokens (sequence, index) that are not there."""
    kd, vd = decoder.decode(cache[0], cache[1]), decoder.decode(cache[2], cache[3])
    ref, bound = np.zeros(qv.shape), np.zeros(qv.shape)
    for b, n in enumerate(lens):
        pg = [table[b, t // page] for t in range(n)]
        for h in range(hq):
            k = np.array([kd[p, h * hkv // hq, t % page] for t, p in enumerate(pg)]).reshape(n, d)
            v = np.array([vd[p, h * hkv // hq, t % page] for t, p in enumerate(pg)]).reshape(n, d)
            for i in range(q_len):
                row = b * q_len + i
                seen = [t for t in range(max(0, n - q_len + 1 + i)) if (b, t) not in hidden]
                r, w, s = decoder.attend(qv[row, h], k, v, seen, scale)
                ref[row, h] = r
                bound[row, h] = attention_bound(r, w, s, len(seen), d, name, EPS_P)
    return ref, bound


def _hold(got, ref, bound):
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {ref[bad][0]} +- {bound[bad][0]}")


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,q_len,hq,hkv,d,page", [
    ([1], 1, 1, 1, 64, 16), ([0, 2, 15], 1, 4, 2, 64, 16), ([16, 17, 31, 33], 1, 8, 1, 128, 16),
    ([63, 64, 65, 128, 129], 1, 6, 2, 128, 48), ([700], 1, 16, 1, 128, 64), ([300, 0, 5], 1, 17, 1, 96, 32),
    ([100, 257], 1, 3, 3, 192, 16), ([90, 190], 1, 10, 2, 256, 128), ([1, 0, 3, 70], 4, 4, 2, 64, 16),
    ([200, 37], 8, 8, 2, 128, 64), ([33, 64], 5, 20, 1, 128, 16), ([12, 300], 16, 6, 2, 96, 16),
    ([2, 40], 3, 64, 1, 256, 16), ([1500, 1, 900], 1, 8, 2, 128, 16)])
def test_decode(lens, q_len, hq, hkv, d, page, name):
    torch = torch_dev()
    rng = np.random.default_rng(sum(lens) + 13 * hq + d)
    table, cache, q, qv = _setup(torch, rng, lens, q_len, hq, hkv, d, page, name)
    ref, bound = _reference(cache, table, lens, qv, q_len, hq, hkv, d, page, d ** -0.5, name)
    for ws in (None, _workspace(torch, lens, q_len, hq, hkv, d, table, page)):
        got = host(_call(torch, q, cache, table, lens, d ** -0.5, ws))
        _hold(got, ref, bound)
        assert (host(_call(torch, q, cache, table, lens, d ** -0.5, ws)) == got).all(), "not the same twice"


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_decode_long_axis_is_split(d, name):
    """A few rows over a long axis, some of its parts with nothing that counts:
    scores so far apart that most probabilities vanish."""
    torch = torch_dev()
    rng = np.random.default_rng(d)
    lens, hq, hkv, page = [9000, 4100], 4, 1, 64
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, name, gain=6.0)
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, name)
    ws = _workspace(torch, lens, 1, hq, hkv, d, table, page)
    for n in (ws.numel(), ws.numel() // 2, 40000, 16):
        got = host(_call(torch, q, cache, table, lens, d ** -0.5, ws[:n]))
        _hold(got, ref, bound)


def test_decode_pages_that_are_not_there():
    """Entries outside the cache hide their tokens, a row may lose all of them;
    lengths past the table read what the table has, negative ones nothing."""
    torch = torch_dev()
    rng = np.random.default_rng(21)
    lens, hq, hkv, d, page = [100, 40, 64, 30], 4, 2, 128, 16
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, "bf16")
    hidden = {(0, t) for t in range(32, 48)} | {(1, t) for t in range(40)}
    cut = table.copy()
    cut[0, 2] = -1
    cut[1, :3] = [cache[0].shape[0], -5, 2 ** 31 - 1]
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, 0.1, "bf16", hidden)
    given = list(lens)
    given[2], given[3] = 64, -3
    ref[3] = bound[3] = 0
    _hold(host(_call(torch, q, cache, cut, given, 0.1)), ref, bound)
    # a table of exactly four pages and a length beyond it
    ref, bound = _reference(cache, table[2:3, :4], [64], qv[2:3], 1, hq, hkv, d, page, 0.1, "bf16")
    _hold(host(_call(torch, q[2:3], cache, np.ascontiguousarray(table[2:3, :4]), [2 ** 31 - 1], 0.1)), ref, bound)


@pytest.mark.parametrize("which", [1, 3])
def test_decode_not_a_number_reaches_only_who_sees_it(which):
    """A token whose keys or values are NaN: rows that see it are NaN (for values:
    in the dimensions of that group), earlier queries and other sequences are not."""
    torch = torch_dev()
    rng = np.random.default_rng(22)
    lens, q_len, hq, hkv, d, page = [70, 50], 4, 4, 2, 128, 16
    table, cache, q, qv = _setup(torch, rng, lens, q_len, hq, hkv, d, page, "bf16")
    ref, bound = _reference(cache, table, lens, qv, q_len, hq, hkv, d, page, 0.1, "bf16")
    t = 68                                                     # queries 2 and 3 of sequence 0 see it
    cache[which][table[0, t // page], 1, t % page, 2] = 255
    got = host(_call(torch, q, cache, table, lens, 0.1))
    hit = np.zeros(got.shape, bool)
    hit[2:4, 2:, 64:96] = True
    if which == 1:
        hit[2:4, 2:] = True
    assert np.isnan(got[hit]).all()
    _hold(got[~hit], ref[~hit], bound[~hit])


def test_decode_strided_queries_and_scores_of_any_size():
    torch = torch_dev()
    rng = np.random.default_rng(23)
    lens, hq, hkv, d, page = [77, 200], 6, 2, 64, 16
    table, cache, _, _ = _setup(torch, rng, lens, 1, hq, hkv, d, page, "fp16")
    big, bv = half(torch, rng.normal(0, 1, (2, hq + 5, d)), "fp16")
    for scale in (0.0, -0.3, 40.0):
        ref, bound = _reference(cache, table, lens, bv[:, 3:3 + hq], 1, hq, hkv, d, page, scale, "fp16")
        _hold(host(_call(torch, big[:, 3:3 + hq], cache, table, lens, scale)), ref, bound)


def test_decode_past_four_gigabytes():
    """Pages whose bytes lie beyond 2^32 of the cache's start."""
    torch = torch_dev()
    rng = np.random.default_rng(24)
    d, hkv, page, hq = 256, 8, 128, 16
    pages = (9 << 29) // (hkv * page * d // 2)
    small = 3
    lens = [300]
    table = np.array([[2, 0, 1]], np.int32)
    kc, vc = (rng.integers(0, 256, (small, hkv, page, d // 2), dtype=np.uint8) for _ in range(2))
    ks, vs = (rng.integers(124, 129, (small, hkv, page, d // 32), dtype=np.uint8) for _ in range(2))
    big = []
    for c in (kc, ks, vc, vs):
        t = torch.empty((pages,) + c.shape[1:], dtype=torch.uint8, device="cuda")
        t[pages - small:] = torch.from_numpy(c).cuda()
        big.append(t)
    assert big[0].numel() > 1 << 32
    q, qv = half(torch, rng.normal(0, 1, (1, hq, d)), "bf16")
    ref, bound = _reference((kc, ks, vc, vs), table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, "bf16")
    out = torch.zeros_like(q)
    W.kv4_attention(q, tuple(big), torch.from_numpy(table + pages - small).cuda(),
                    torch.tensor(lens, dtype=torch.int32, device="cuda"), out, d ** -0.5)
    _hold(host(out), ref, bound)


def test_decode_on_another_stream_and_in_a_graph():
    """A captured append and attention, replayed over changing tokens with eager
    work between the replays, against the same calls made eagerly."""
    torch = torch_dev()
    rng = np.random.default_rng(25)
    lens, hq, hkv, d, page = [2000, 333], 8, 2, 128, 64
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, "bf16")
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, "bf16")
    ws = _workspace(torch, lens, 1, hq, hkv, d, table, page)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = _call(torch, q, cache, table, lens, d ** -0.5, ws)
    side.synchronize()
    _hold(host(got), ref, bound)

    dev = tuple(torch.from_numpy(c).cuda() for c in cache)
    tab, n = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    cs = torch.zeros((1, 0), device="cuda")
    k, v = (torch.zeros((2, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    slots = torch.tensor([int(table[b, (m - 1) // page]) * page + (m - 1) % page for b, m in enumerate(lens)],
                         device="cuda")
    qt, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        W.kv4_append(q, k, v, cs, pos, slots, dev, qt)
        W.kv4_attention(qt, dev, tab, n, out, d ** -0.5, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(half(torch, rng.normal(0, 1 + i, tuple(t.shape)), "bf16")[0])
        ws.fill_(255)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        one = out.clone()
        ws.fill_(i)
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(one, out) and float(one.abs().sum()) > 0


def test_decode_empty_batches():
    torch = torch_dev()
    rng = np.random.default_rng(26)
    table, cache, q, qv = _setup(torch, rng, [5], 1, 2, 1, 64, 16, "bf16")
    dev = tuple(torch.from_numpy(c).cuda() for c in cache)
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    W.kv4_attention(none, dev, torch.zeros((0, 3), **i32), torch.zeros(0, **i32), none.clone(), 1.0)
    out = torch.full_like(q, 5.0)
    W.kv4_attention(q, dev, torch.zeros((1, 0), **i32), torch.tensor([7], **i32), out, 1.0)     # a table of no pages
    assert (out == 0).all()


def test_decode_refuses_other_tensors():
    torch = torch_dev()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731

    def cache(d=64, page=16, hkv=2):
        return tuple(z(3, hkv, page, w, dt=torch.uint8) for w in (d // 2, d // 32, d // 2, d // 32))

    q, c, t, n = z(2, 4, 64), cache(), z(2, 2, dt=torch.int32), z(2, dt=torch.int32)
    W.kv4_attention(q, c, t, n, z(2, 4, 64), 1.0)
    for bad in (lambda: W.kv4_attention(q.float(), c, t, n, q, 1.0), lambda: W.kv4_attention(q, c, t.long(), n, q, 1.0),
                lambda: W.kv4_attention(q, c, t, n[:1], q, 1.0), lambda: W.kv4_attention(q, c, t, n, q[:1], 1.0),
                lambda: W.kv4_attention(z(3, 4, 64), c, t, n, z(3, 4, 64), 1.0),
                lambda: W.kv4_attention(z(2, 4, 128), c, t, n, z(2, 4, 128), 1.0),
                lambda: W.kv4_attention(q, c[:2] + cache(hkv=1)[2:], t, n, q, 1.0),
                lambda: W.kv4_attention(q, c, t, n, z(2, 4, 64).half(), 1.0),
                lambda: W.kv4_attention(q, c, t, n, z(2, 4, 64), 1.0, workspace=torch.zeros(64))):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: W.kv4_attention(z(2, 3, 64), c, t, n, z(2, 3, 64), 1.0), -1),
                        (lambda: W.kv4_attention(q, c, t, n, z(2, 4, 64), float("nan")), -1),
                        (lambda: W.kv4_attention(q, c, t, n, z(2, 4, 64), float("inf")), -1),
                        (lambda: W.kv4_attention(z(2, 4, 32), cache(32), t, n, z(2, 4, 32), 1.0), -2),
                        (lambda: W.kv4_attention(q, cache(page=8), t, n, z(2, 4, 64), 1.0), -2)):
        with pytest.raises(W.WinoError) as e:
            bad()
        assert e.value.status == status

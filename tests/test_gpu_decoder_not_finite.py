"""Queries, keys and values that are not finite, on the paths of the decoder
operators where the parts of a row meet: a row that sees a NaN is NaN however
its work was shared out, every other row has its ordinary result (the bounds
are those of the operators' own tests)."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from decoder_util import half, host
from gpu_util import torch_dev
from test_gpu_kv4_attention import _call, _hold, _reference, _setup, _workspace
from test_gpu_prompt_attention import _cu
from test_gpu_prompt_attention import _reference as prompt_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_split_decode_keeps_a_query_that_is_not_a_number(d, name):
    """All scores of such a row are NaN, in each of its parts."""
    torch = torch_dev()
    rng = np.random.default_rng(d)
    lens, hq, hkv, page = [4000, 0, 700], 4, 2, 64
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, name)
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, name)
    hit = np.zeros((3, hq), bool)
    hit[0, 1] = hit[2, 3] = True
    q[0, 1, d - 3] = q[2, 3] = q[1, 2] = float("nan")             # sequence 1 has no tokens: zeros all the same
    ws = _workspace(torch, lens, 1, hq, hkv, d, table, page)
    assert ws.numel() > 16
    for w in (None, ws):
        got = host(_call(torch, q, cache, table, lens, d ** -0.5, w))
        assert np.isnan(got[hit]).all()
        _hold(got[~hit], ref[~hit], bound[~hit])


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("length,begins", [(2817, [2816, 2304, 1000, 0]), (2561, [2560, 2048, 768, 256])])
def test_split_decode_keeps_keys_that_are_not_numbers(length, begins, name):
    """Runs of such keys to the end of a sequence, some of them exactly one part or several; the sequence beside it
    has its ordinary result."""
    torch = torch_dev()
    rng = np.random.default_rng(length)
    lens, hq, hkv, d, page = [length, 900], 3, 1, 128, 64
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, name)
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, name)
    ws = _workspace(torch, lens, 1, hq, hkv, d, table, page)
    assert ws.numel() > 16
    sound = cache[1].copy()
    for begin in begins:
        cache[1][:] = sound
        for t in range(begin, length):
            cache[1][table[0, t // page], 0, t % page, 1] = 255
        for w in (None, ws):
            got = host(_call(torch, q, cache, table, lens, d ** -0.5, w))
            assert np.isnan(got[0]).all(), f"keys from {begin} on"
            _hold(got[1], ref[1], bound[1])


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,hq,hkv,d", [([5, 40], 4, 2, 64), ([3, 70], 2, 1, 96), ([200, 90], 3, 1, 128), ([700], 16, 16, 256),
                                           ([1100, 3], 12, 12, 192)])
def test_prompt_scores_that_are_all_minus_infinity(lens, hq, hkv, d, name):
    """A row that sees keys, each of them infinitely far away, is not a number: its softmax is infinity less itself.
    A row that sees no key is zeros, whatever its query."""
    torch = torch_dev()
    rng = np.random.default_rng(d)
    k_lens = [n - 2 for n in lens]                                       # the first two rows of a sequence see nothing
    qn, kn = sum(lens), sum(k_lens)
    q, qv = half(torch, rng.normal(0, 1, (qn, hq, d)), name)
    k, kv = half(torch, rng.normal(0, 1, (kn, hkv, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (kn, hkv, d)), name)
    k[:, :, 7] = -k[:, :, 7].abs() - 0.5
    kv = host(k)
    rows = [0, 1, 2, lens[0] - 1, qn - 1]
    ref, bound = prompt_reference(qv, kv, vv, lens, k_lens, d ** -0.5, True, name) if qn < 300 else (None, None)
    for r in rows:
        q[r, hq - 1, 7] = float("inf")
    out = torch.full_like(q, 3.0)
    W.prompt_attention(q, k, v, _cu(torch, lens), _cu(torch, k_lens), max(lens), out, d ** -0.5)
    got = host(out)
    hit = np.zeros((qn, hq), bool)
    hit[rows, hq - 1] = True
    blind = np.zeros((qn, hq), bool)
    for b in np.cumsum([0] + lens[:-1]):
        blind[b:b + 2] = True
    assert (got[blind] == 0).all()
    assert np.isnan(got[hit & ~blind]).all()
    assert np.isfinite(got[~hit]).all()
    if ref is not None:
        _hold(got[~hit], ref[~hit], bound[~hit])


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_decode_scores_that_are_all_minus_infinity(d, name):
    """An infinite query on keys that are all negative there, in sequences of one token to many parts: not a number
    where any token is seen, zeros where none is (an empty sequence, pages that are not there)."""
    torch = torch_dev()
    rng = np.random.default_rng(d + 3)
    lens, hq, hkv, page = [1, 30, 3000, 0, 40], 5, 1, 16
    table, cache, q, qv = _setup(torch, rng, lens, 1, hq, hkv, d, page, name)
    cache[0][..., 3] |= 0xB0                                      # dimension 7: -3 to -6
    table[4, :3] = -1
    hidden = {(4, t) for t in range(40)}
    ref, bound = _reference(cache, table, lens, qv, 1, hq, hkv, d, page, d ** -0.5, name, hidden)
    hit = np.zeros((5, hq), bool)
    hit[:, 2] = hit[2, 4] = True
    q[torch.from_numpy(hit).cuda(), 7] = float("inf")
    ws = _workspace(torch, lens, 1, hq, hkv, d, table, page)
    assert ws.numel() > 16
    for w in (None, ws):
        got = host(_call(torch, q, cache, table, lens, d ** -0.5, w))
        assert np.isnan(got[:3][hit[:3]]).all() and (got[3:] == 0).all()
        _hold(got[~hit], ref[~hit], bound[~hit])

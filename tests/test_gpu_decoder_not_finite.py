"""Queries, keys and values that are not finite, on the paths of the decoder
operators where the parts of a row meet: a row that sees a NaN is NaN however
its work was shared out, every other row has its ordinary result (the bounds
are those of the operators' own tests)."""
import numpy as np
import pytest

from decoder_util import host
from gpu_util import torch_dev
from test_gpu_kv4_attention import _call, _hold, _reference, _setup, _workspace

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

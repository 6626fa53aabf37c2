"""CPU-side checks of the 4-bit decoder operators: the weight quantizer against
the oracle, the oracle's format against its definition, and refusals that need
no device."""
import ctypes

import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder


def _lib():
    try:
        return W.load_library()
    except W.LibraryNotBuilt:
        pytest.skip("library not built")


def test_quantizer_matches_oracle():
    _lib()
    rng = np.random.default_rng(1)
    w = (rng.normal(0, 1, (9, 160)) * np.exp2(rng.integers(-20, 20, (9, 160)) * (rng.random((9, 1)) < 0.5))).astype(np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    w[0, :32] = np.tile(np.concatenate([ties, -ties]), 2) * 2.0 ** -9
    w[1, :32] = 0
    w[2, :32] = np.float32(1e-44) * np.arange(32)
    w[3, :32] = 3.4e38
    w[4, :32] = 6.0 * 2.0 ** 7
    w[5, :32] = np.nextafter(np.float32(6.0), np.float32(7.0))
    codes, scales = W.w4_quantize_weights(w)
    rc, rs = decoder.encode(w)
    assert (codes == rc).all() and (scales == rs).all()


def test_quantizer_edges():
    lib = _lib()
    codes, scales = W.w4_quantize_weights(np.zeros((0, 64), np.float32))
    assert codes.shape == (0, 32) and scales.shape == (0, 2)
    with pytest.raises(W.WinoError):
        W.w4_quantize_weights(np.zeros((2, 40), np.float32))
    bad = np.zeros((1, 32), np.float32)
    for v in (np.nan, np.inf):
        bad[0, 3] = v
        with pytest.raises(W.WinoError):
            W.w4_quantize_weights(bad)
    assert lib.w4_quantize_weights(None, 1, 32, None, None) == -1


def test_quantizer_picks_the_nearest_value():
    """Every value within the range of its scale is off by at most half the gap to
    its neighbours, and the scale is the smallest that holds the maximum."""
    rng = np.random.default_rng(2)
    x = rng.normal(0, 3, (50, 64))
    c, s = decoder.encode(x)
    e = s.astype(int) - 127
    g = np.abs(x).reshape(50, 2, 32).max(-1)
    assert (g <= 6 * 2.0 ** e).all() and (g > 6 * 2.0 ** (e - 1)).all()
    a = np.abs(x) * np.repeat(2.0 ** -e, 32, -1)
    gap = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    err = np.abs(decoder.decode(c, s) - x) * np.repeat(2.0 ** -e, 32, -1)
    assert (err <= gap / 2).all()


def test_refusals_without_a_device():
    lib = _lib()
    a = np.zeros(4096, np.uint8)
    p = (a.ctypes.data + 63) // 64 * 64                  # never read

    def matvec(x=p, xs=64, codes=p, scales=p, bias=None, y=p, ys=8, m=2, n=8, k=64, kind=0, ws=None, wb=0):
        return lib.w4_matvec(x, xs, codes, scales, bias, y, ys, m, n, k, kind, ws, wb, None)

    for kw, want in (({"kind": 2}, -1), ({"x": None}, -1), ({"codes": None}, -1), ({"scales": None}, -1),
                     ({"y": None}, -1), ({"m": -1}, -1), ({"n": -1}, -1), ({"k": 48}, -1), ({"k": -32}, -1),
                     ({"xs": 63}, -1), ({"ys": 7}, -1), ({"xs": 68}, -2), ({"x": p + 8}, -2), ({"codes": p + 4}, -2),
                     ({"m": 70000}, -2), ({"k": 1 << 21, "xs": 1 << 21}, -2), ({"m": 0}, 0), ({"n": 0}, 0)):
        assert matvec(**kw) == want, kw
    assert W.w4_matvec_workspace_bytes(-1, 5, 64) == 0

    def cache(**kw):
        f = dict(k_codes=p, k_scales=p, v_codes=p, v_scales=p, pages=2, kv_heads=2, page_size=16, head_dim=64)
        f.update(kw)
        return ctypes.byref(W.binding._KV4Cache(**f))

    def append(q=p, qs=256, k=p, ks=128, v=p, vs=128, t=2, h=4, cs=p, rows=4, rot=64, pos=p, slots=p, c=None, qo=p,
               ko=None, vo=None, rotary=0, values=0, kind=0):
        return lib.kv4_append(q, qs, k, ks, v, vs, t, h, cs, rows, rot, pos, slots, cache() if c is None else c, qo, ko,
                              vo, rotary, values, kind, None)

    for kw, want in (({"kind": -1}, -1), ({"rotary": 2}, -1), ({"values": 2}, -1), ({"k": None}, -1), ({"v": None}, -1),
                     ({"q": None}, -1), ({"qo": None}, -1), ({"h": 0}, -1), ({"pos": None}, -1), ({"slots": None}, -1),
                     ({"cs": None}, -1), ({"t": -1}, -1), ({"rot": 128}, -1), ({"rot": 24}, -2), ({"qs": 255}, -1),
                     ({"ks": 120}, -1), ({"ks": 132}, -2), ({"k": p + 2}, -2), ({"cs": p + 4}, -2),
                     ({"c": cache(page_size=24)}, -2), ({"c": cache(head_dim=80)}, -2), ({"c": cache(pages=-1)}, -1),
                     ({"c": cache(k_scales=None)}, -1), ({"c": cache(kv_heads=0)}, -1), ({"c": cache(v_codes=p + 2)}, -2),
                     ({"c": cache(head_dim=288), "qs": 2000, "ks": 600, "vs": 600}, -2), ({"t": 0}, 0)):
        assert append(**kw) == want, kw
    assert lib.kv4_append(p, 256, p, 128, p, 128, 1, 4, p, 4, 64, p, p, None, p, None, None, 0, 0, 0, None) == -1

    def attention(q=p, qs=256, c=None, table=p, mp=2, lens=p, out=p, b=2, ql=1, h=4, scale=1.0, kind=0, ws=None, wb=0):
        return lib.kv4_attention(q, qs, cache() if c is None else c, table, mp, lens, out, b, ql, h, scale, kind, ws, wb,
                                 None)

    for kw, want in (({"kind": 3}, -1), ({"q": None}, -1), ({"table": None}, -1), ({"lens": None}, -1), ({"out": None}, -1),
                     ({"h": 3}, -1), ({"h": 0}, -1), ({"b": -1}, -1), ({"ql": -1}, -1), ({"mp": -1}, -1),
                     ({"scale": float("nan")}, -1), ({"scale": float("-inf")}, -1), ({"qs": 255}, -1), ({"qs": 260}, -2),
                     ({"q": p + 8}, -2), ({"c": cache(head_dim=32)}, -2), ({"c": cache(page_size=20)}, -2),
                     ({"c": cache(v_scales=None)}, -1), ({"b": 1 << 30, "ql": 1 << 20}, -2), ({"b": 0}, 0), ({"ql": 0}, 0)):
        assert attention(**kw) == want, kw
    assert W.kv4_attention_workspace_bytes(-1, 1, 4, 2, 64, 2, 16) == 0

    def prompt(q=p, qs=256, k=p, ks=128, v=p, vs=128, cq=p, ck=p, seqs=1, tq=4, tk=4, mq=4, h=4, hkv=2, d=64, scale=1.0,
               causal=1, out=p, kind=0):
        return lib.prompt_attention(q, qs, k, ks, v, vs, cq, ck, seqs, tq, tk, mq, h, hkv, d, scale, causal, out, kind, None)

    for kw, want in (({"kind": 2}, -1), ({"q": None}, -1), ({"k": None}, -1), ({"v": None}, -1), ({"out": None}, -1),
                     ({"cq": None}, -1), ({"ck": None}, -1), ({"seqs": -1}, -1), ({"tq": -1}, -1), ({"tk": -1}, -1),
                     ({"mq": -1}, -1), ({"h": 5}, -1), ({"hkv": 0}, -1), ({"causal": 2}, -1), ({"d": 80}, -2), ({"d": 0}, -1),
                     ({"scale": float("nan")}, -1), ({"qs": 200}, -1), ({"ks": 100}, -1), ({"vs": 100}, -1),
                     ({"vs": 132}, -2), ({"v": p + 4}, -2), ({"tq": 0}, 0)):
        assert prompt(**kw) == want, kw


def test_append_of_no_tokens_needs_no_addresses():
    """An empty tensor's address may be null: queries of no tokens are no reason to refuse."""
    lib = _lib()
    c = W.binding._KV4Cache(k_codes=64, k_scales=64, v_codes=64, v_scales=64, pages=2, kv_heads=2, page_size=16, head_dim=64)
    for heads in (0, 4):
        assert lib.kv4_append(None, 256, None, 128, None, 128, 0, heads, None, 0, 64, None, None, ctypes.byref(c), None,
                              None, None, 0, 0, 0, None) == 0


def test_matvec_parts_count_the_rows_of_x():
    """k is cut into parts only to make 256 workgroups of 64 x 64 results at most; many rows of x are workgroups
    enough, so the parts' sums never need more than their 4 MiB."""
    _lib()
    for n in (40, 1000, 4096, 4100, 8192, 16384):
        for k in (1024, 4096, 8192, 16384, 1 << 20):
            for m in (1, 16, 17, 64, 65, 130, 512, 2048, 8192, 65535):
                assert W.w4_matvec_workspace_bytes(m, n, k) <= 4 << 20, (m, n, k)
    assert W.w4_matvec_workspace_bytes(64, 4096, 16384) > 0          # a few rows still are cut
    assert W.w4_matvec_workspace_bytes(128, 1024, 16384) > 0


def test_matvec_parts_do_not_end_beside_a_size():
    """A long k of few outputs is shared out to workgroups whatever the number of outputs: one more than a round
    number of tiles is no reason to leave half of the device idle."""
    _lib()
    for m in (4, 8, 9, 12, 16, 48):
        for n in (1024, 2560, 3584, 4000, 4095, 4096, 4097, 4128, 4160, 5003, 5120, 6000):
            assert W.w4_matvec_workspace_bytes(m, n, 16384) > 0, (m, n)


def test_matvec_sizes_that_are_refused_need_no_workspace():
    _lib()
    top = 2 ** 31 - 1
    for a in ((65536, 4096, 16384), (16, (1 << 24) + 1, 4096), (16, 64, (1 << 20) + 32), (top, top, top), (1, top, 8192)):
        assert W.w4_matvec_workspace_bytes(*a) == 0, a


def test_attention_of_more_rows_than_a_launch_holds():
    """A launch has less than 2^32 threads, 512 for each sequence and set of 16 rows: more is refused before anything
    is launched, and rows that the join could not hold (256 threads each) are not split."""
    lib = _lib()
    c = W.binding._KV4Cache(k_codes=64, k_scales=64, v_codes=64, v_scales=64, pages=2, kv_heads=2, page_size=16, head_dim=64)
    for batch, q_len, heads in ((1 << 22, 1, 2), (1 << 21, 20, 4), ((1 << 23) - 1, 1, 16)):
        assert lib.kv4_attention(64, 64 * heads, ctypes.byref(c), 64, 2, 64, 64, batch, q_len, heads, 1.0, 0, None, 0,
                                 None) == -2, (batch, q_len, heads)
    assert W.kv4_attention_workspace_bytes(2, 1, 32, 8, 128, 2048, 64) > 0
    assert W.kv4_attention_workspace_bytes(1 << 17, 1, 128, 8, 128, 2048, 64) == 0


def test_prompt_of_more_sequences_than_a_launch_holds():
    lib = _lib()
    for d, heads, kv_heads in ((64, 256, 256), (256, 128, 128), (192, 1024, 256)):
        assert lib.prompt_attention(64, heads * d, 64, kv_heads * d, 64, kv_heads * d, 64, 64, 65536, 64, 64, 1, heads,
                                    kv_heads, d, 1.0, 1, 64, 0, None) == -2, (d, heads)

"""CPU-side checks of the 8-bit decoder operators: refusals that need no device,
the quantizer's arithmetic, and the oracle against its definition."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder8


def _lib():
    try:
        return W.load_library()
    except W.LibraryNotBuilt:
        pytest.skip("library not built")


def _address():
    a = np.zeros(4096, np.uint8)
    return a, (a.ctypes.data + 63) // 64 * 64                # never read


def test_quantize_refusals():
    lib = _lib()
    keep, p = _address()

    def call(x=p, xs=64, codes=p, scales=p, m=2, k=64, kind=0):
        return lib.w8_quantize(x, xs, codes, scales, m, k, kind, None)

    for kw, want in (({"kind": 2}, -1), ({"kind": -1}, -1), ({"m": -1}, -1), ({"k": -16}, -1), ({"k": 40}, -1), ({"x": None}, -1),
                     ({"codes": None}, -1), ({"scales": None}, -1), ({"xs": 48}, -1), ({"xs": 68}, -2), ({"x": p + 8}, -2),
                     ({"codes": p + 8}, -2), ({"scales": p + 2}, -2), ({"m": 1 << 24}, -2), ({"m": 0}, 0), ({"m": 0, "x": None}, 0)):
        assert call(**kw) == want, kw


def test_matmul_refusals():
    lib = _lib()
    keep, p = _address()

    def call(x=p, xs=64, sx=p, w=p, sw=p, bias=None, y=p, ys=8, m=2, n=8, k=64, kind=0, ws=None, wb=0):
        return lib.w8_matmul(x, xs, sx, w, sw, bias, y, ys, m, n, k, kind, ws, wb, None)

    for kw, want in (({"kind": 2}, -1), ({"x": None}, -1), ({"sx": None}, -1), ({"w": None}, -1), ({"sw": None}, -1),
                     ({"y": None}, -1), ({"m": -1}, -1), ({"n": -1}, -1), ({"k": -16}, -1), ({"k": 24}, -1), ({"xs": 48}, -1),
                     ({"ys": 7}, -1), ({"xs": 72}, -2), ({"x": p + 8}, -2), ({"w": p + 4}, -2), ({"sx": p + 2}, -2),
                     ({"sw": p + 1}, -2), ({"y": p + 1}, -2), ({"bias": p + 1}, -2), ({"ws": p + 8}, -2),
                     ({"k": 1 << 17, "xs": 1 << 17}, -2), ({"m": (1 << 20) + 1}, -2), ({"n": (1 << 24) + 1, "ys": 1 << 25}, -2),
                     ({"m": 1 << 20, "n": 1 << 24, "ys": 1 << 24}, -2), ({"m": 0}, 0), ({"n": 0}, 0)):
        assert call(**kw) == want, kw
    assert W.w8_matmul_workspace_bytes(-1, 5, 64) == 0
    assert W.w8_matmul_workspace_bytes(5, 5, 1 << 17) == 0


def test_route_refusals():
    lib = _lib()
    keep, p = _address()

    def call(logits=p, stride=8, bias=None, t=2, e=8, top=2, score=0, g=1, tg=1, best=1, norm=1, scale=1.0, live=None, chosen=p,
             weights=p, order=p, ends=p, kind=0, ws=p, wb=4096):
        return lib.route_experts(logits, stride, bias, t, e, top, score, g, tg, best, norm, scale, live, chosen, weights, order,
                                 ends, kind, ws, wb, None)

    need = W.route_experts_workspace_bytes(65, 8, 2)
    assert need > 0 and W.route_experts_workspace_bytes(32, 8, 2) == 0
    for kw, want in (({"kind": 3}, -1), ({"kind": -1}, -1), ({"score": 2}, -1), ({"t": -1}, -1), ({"e": 0}, -1), ({"top": 0}, -1),
                     ({"top": 9}, -1), ({"g": 0}, -1), ({"g": 3}, -1), ({"g": 4, "tg": 5}, -1), ({"tg": 0}, -1),
                     ({"g": 4, "tg": 2, "top": 5}, -1), ({"best": 0}, -1), ({"best": 3}, -1), ({"g": 8, "tg": 2, "best": 2}, -1),
                     ({"norm": 2}, -1), ({"scale": float("nan")}, -1), ({"scale": float("inf")}, -1), ({"order": None}, -1),
                     ({"ends": None}, -1), ({"logits": None}, -1), ({"chosen": None}, -1), ({"weights": None}, -1),
                     ({"stride": 7}, -1), ({"t": 65, "ws": None}, -1), ({"t": 65, "wb": need - 1}, -1), ({"e": 1025, "stride": 1025}, -2),
                     ({"e": 128, "stride": 128, "top": 33}, -2), ({"e": 130, "stride": 130, "g": 65}, -2),
                     ({"t": 1 << 22}, -2), ({"logits": p + 1}, -2), ({"kind": 2, "logits": p + 2}, -2), ({"bias": p + 2}, -2),
                     ({"live": p + 2}, -2), ({"chosen": p + 2}, -2), ({"weights": p + 1}, -2), ({"order": p + 2}, -2),
                     ({"ends": p + 2}, -2), ({"ws": p + 2}, -2), ({"t": 0, "order": None, "ends": None}, 0)):
        assert call(**kw) == want, kw
    assert W.route_experts_workspace_bytes(-1, 8, 2) == 0
    assert W.route_experts_workspace_bytes(4, 2000, 2) == 0


def test_experts_refusals():
    lib = _lib()
    keep, p = _address()

    def call(x=p, xs=64, sx=p, rows=2, w=p, sw=p, order=p, ends=p, routes=4, e=3, chosen=None, weights=None, top=1, y=p, ys=8, n=8,
             k=64, kind=0, ws=p, wb=4096):
        return lib.w8_experts_matmul(x, xs, sx, rows, w, sw, order, ends, routes, e, chosen, weights, top, y, ys, n, k, kind, ws, wb,
                                     None)

    for kw, want in (({"kind": 2}, -1), ({"rows": -1}, -1), ({"rows": 0}, -1), ({"rows": 3}, -1), ({"routes": -1}, -1), ({"e": 0}, -1),
                     ({"n": -1}, -1), ({"k": 24}, -1), ({"k": -16}, -1), ({"chosen": p}, -1), ({"weights": p}, -1),
                     ({"chosen": p, "weights": p, "top": 0}, -1), ({"chosen": p, "weights": p, "top": 3}, -1),
                     ({"chosen": p, "weights": p, "top": 2, "ws": None}, -1), ({"chosen": p, "weights": p, "top": 2, "wb": 64}, -1),
                     ({"x": None}, -1), ({"sx": None}, -1), ({"w": None}, -1), ({"sw": None}, -1), ({"order": None}, -1),
                     ({"ends": None}, -1), ({"y": None}, -1), ({"xs": 48}, -1), ({"ys": 7}, -1), ({"xs": 72}, -2),
                     ({"x": p + 8}, -2), ({"w": p + 8}, -2), ({"sx": p + 2}, -2), ({"sw": p + 2}, -2), ({"order": p + 2}, -2),
                     ({"ends": p + 2}, -2), ({"y": p + 1}, -2), ({"ws": p + 8}, -2), ({"e": 1025}, -2), ({"k": 1 << 17, "xs": 1 << 17}, -2),
                     ({"routes": (1 << 22) + 2}, -2), ({"n": (1 << 20) + 1, "ys": 1 << 21}, -2),
                     ({"routes": 1 << 22, "rows": 1 << 22, "n": 1 << 20, "ys": 1 << 20}, -2),
                     ({"routes": 1 << 17, "rows": 1 << 17, "e": 100, "xs": 1 << 17, "n": 900000, "ys": 900000, "k": 16}, -2),
                     ({"routes": 0}, 0), ({"n": 0}, 0)):
        assert call(**kw) == want, kw
    assert W.w8_experts_matmul_workspace_bytes(-1, 8, 1) == 0
    assert W.w8_experts_matmul_workspace_bytes(4, 8, 0) == 0


@pytest.mark.parametrize("bits", [8, 11])
def test_quantizer_arithmetic(bits):
    """The kernel's fp32 steps give R(127 x / a) for all significands of x <= a: q = x (127 / a), raised by 2^-21 of its
    magnitude, floor(q + 1/2).  Quotients below 1/4 give 0 whatever their last bits."""
    f = np.float32
    sig = np.arange(1 << (bits - 1), 1 << bits, dtype=np.int64)
    # every sixteenth a of fp16, and the ends of the range
    tops = sig if bits == 8 else np.concatenate([sig[::16], sig[-3:], [1025, 1027]])
    for a in tops:
        for d in range(9):                                   # x = X 2^-d
            x = sig if d else sig[sig <= a]
            exact = (2 * 127 * x + a * 2 ** d) // (2 * a * 2 ** d), (-2 * 127 * x + a * 2 ** d) // (2 * a * 2 ** d)
            inv = f(127) / f(a)
            for sign, want in zip((1, -1), exact):
                q = (f(sign) * x.astype(f) * f(2.0 ** -d)) * inv
                q = (np.abs(q).astype(np.float64) * 2.0 ** -21 + q.astype(np.float64)).astype(f)     # one rounding
                assert (np.floor(q + f(0.5)) == want).all(), (a, d, sign)


def test_oracle_quantizer():
    rng = np.random.default_rng(5)
    x = rng.normal(0, 2, 300)
    codes, scale = decoder8.quantize_row(x)
    assert np.abs(codes).max() == 127
    assert (np.abs(codes * float(scale) - x) <= float(scale) * (0.5 + 1e-12)).all()
    codes, scale = decoder8.quantize_row([2.0, 1.0, -1.0, -2.0, 0.0])     # 63.5 goes up, so does -63.5
    assert list(codes) == [127, 64, -63, -127, 0]


def test_oracle_route():
    s = np.array([0.1, 0.3, 0.3, 0.05, 0.15, 0.1])
    assert decoder8.route_row(s, None, 3, 1, 1, 1) == [1, 2, 4]
    assert decoder8.route_row(s, None, 2, 3, 1, 2) == [1, 0]               # pairs: 0.4, 0.35, 0.25
    assert decoder8.route_row(s, np.array([0, 0, 0, 0, 0, 1.0]), 2, 3, 1, 1) == [5, 4]
    routes, ends = decoder8.order([[2, 0], [0, 2], [-1, 1]], 3)
    assert list(routes) == [1, 2, 5, 0, 3] and list(ends) == [0, 2, 3, 5]

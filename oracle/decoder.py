"""Oracle of the 4-bit decoder operators: the format's definition and the
operators' formulas in float64, written element by element where that is
plainest.  The rotation is done in float32, every product and sum rounded once,
which is how the operator defines it."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])


def scale_byte(amax):
    """e + 127 for the smallest e >= -127 with amax <= 6 * 2^e; 127 for 0, 255
    where amax is not finite."""
    if not np.isfinite(amax):
        return 255
    if amax == 0:
        return 127
    e = -127
    while amax > 6 * 2.0 ** e:
        e += 1
    return e + 127


def code(x, e):
    """The nearest code to x / 2^e: distances to all magnitudes, the even code on a tie."""
    a = abs(float(x)) * 2.0 ** -e
    d = np.abs(MAGNITUDES - a)
    best = np.flatnonzero(d == d.min())
    c = int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])
    return c + (8 if np.signbit(x) else 0)


def encode(x):
    """[..., d] -> codes uint8 [..., d/2], scales uint8 [..., d/32]."""
    x = np.asarray(x)
    flat = x.reshape(-1, 32)
    codes = np.zeros((len(flat), 32), np.uint8)
    scales = np.zeros(len(flat), np.uint8)
    for i, g in enumerate(flat):
        scales[i] = scale_byte(float(np.abs(g.astype(np.float64)).max()) if np.isfinite(g).all() else np.inf)
        if scales[i] != 255:
            codes[i] = [code(v, int(scales[i]) - 127) for v in g]
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales.reshape(*x.shape[:-1], x.shape[-1] // 32)


def decode(codes, scales):
    """float64 values of codes [..., d/2] with scales [..., d/32]."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return VALUES[c] * np.repeat(s, 32, -1)


def rotate(x, cos_sin_rows, pairs):
    """float32 x [tokens, heads, d], cos_sin_rows [tokens, r]: the first r
    dimensions turned; float32 arithmetic, each operation rounded."""
    x = np.asarray(x, np.float32).copy()
    r = cos_sin_rows.shape[1]
    h = r // 2
    j = np.arange(h)
    a, b = (2 * j, 2 * j + 1) if pairs else (j, j + h)
    c, s = cos_sin_rows[:, None, :h].astype(np.float32), cos_sin_rows[:, None, h:].astype(np.float32)
    u, w = x[..., a].copy(), x[..., b].copy()
    x[..., a] = u * c - w * s
    x[..., b] = w * c + u * s
    return x


def attend(q, k, v, visible, scale):
    """One query q [d] over the tokens `visible` of k, v [t, d].  Returns the
    result, sum_t p_t |v_t| and the largest |scale| * sum |q||k| (both for error
    bounds); zeros where nothing is visible."""
    q = np.asarray(q, np.float64)
    d = v.shape[1]
    if len(visible) == 0:
        return np.zeros(d), np.zeros(d), 0.0
    kk, vv = k[visible].astype(np.float64), v[visible].astype(np.float64)
    z = scale * (kk @ q)
    p = np.exp(z - z.max())
    p /= p.sum()
    return p @ vv, p @ np.abs(vv), float(abs(scale) * (np.abs(kk) @ np.abs(q)).max())

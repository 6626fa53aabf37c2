"""Oracle of the 8-bit decoder operators: the formulas in whole numbers,
rationals and float64, written row by row."""
from fractions import Fraction

import numpy as np


def quantize_row(x):
    """float64 values (finite) -> codes and the exact scale max|x| / 127 as a
    Fraction; the code is 127 x / max|x|, halves up."""
    x = [Fraction(float(v)) for v in x]
    top = max((abs(v) for v in x), default=Fraction(0))
    if top == 0:
        return np.zeros(len(x), np.int64), Fraction(0)
    return np.array([(2 * 127 * v + top) // (2 * top) for v in x], np.int64), top / 127


def product(x, x_scales, w, w_scales, bias=None):
    """float64 [m, n] of codes x [m, k], w [n, k] and their scales."""
    sums = x.astype(np.float64) @ w.astype(np.float64).T        # whole numbers below 2^53: exact
    y = sums * np.asarray(x_scales, np.float64)[:, None] * np.asarray(w_scales, np.float64)
    return y if bias is None else y + np.asarray(bias, np.float64)


def scores(logits, sigmoid):
    z = np.asarray(logits, np.float64)
    with np.errstate(all="ignore"):
        if sigmoid:
            return 1 / (1 + np.exp(-z))
        e = np.exp(z - z.max(-1, keepdims=True))
        return e / e.sum(-1, keepdims=True)


def route_row(s, bias, top, groups, top_groups, group_best):
    """Chosen experts of one token with scores s."""
    def number(v):
        return -np.inf if np.isnan(v) else v

    n = len(s) // groups
    with np.errstate(all="ignore"):
        c = [number(v) for v in (s if bias is None else s + np.asarray(bias, np.float64))]
        kept = range(groups)
        if top_groups < groups:
            value = [number(np.sum(sorted(c[g * n:g * n + n], reverse=True)[:group_best])) for g in range(groups)]
            kept = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
    there = [e for e in range(len(s)) if e // n in kept]
    return sorted(there, key=lambda e: (-c[e], e))[:top]


def weights(s, chosen, normalise, scale):
    w = s[chosen]
    if normalise:
        total = w.sum()
        w = w * 0 if total == 0 else w / total
    return w * scale


def order(chosen, experts):
    """Routes by expert and where each expert's begin; what is no expert is left out."""
    flat = np.asarray(chosen).reshape(-1)
    by = [np.flatnonzero(flat == e) for e in range(experts)]
    return np.concatenate(by), np.concatenate([[0], np.cumsum([len(r) for r in by])])


def experts_product(x, x_scales, w, w_scales, routes, ends, total):
    """float64 [total, n], NaN where a route is not in the order."""
    y = np.full((total, w.shape[1]), np.nan)
    share = total // len(x)
    for e in range(len(w)):
        r = np.asarray(routes[ends[e]:ends[e + 1]])
        y[r] = product(x[r // share], x_scales[r // share], w[e], w_scales[e])
    return y

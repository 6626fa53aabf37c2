"""route_experts against the oracle in float64: the choice and the order are
equal.  A weight is off by one rounding to fp32 (2^-24 of itself) and by what 64
bits lose in exponentials, sums of up to 1024 of them and quotients (below 2^-40).

Random choices are equal although the oracle's exponentials may differ from the
kernel's in the last place: values would have to lie within 2^-50 of each other
without being equal, and equal logits give equal values on both sides."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder8

from gpu_util import torch_dev

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "fp16", "fp32"]


def run(torch, logits, top, bias=None, live=None, ordered=True, **how):
    t, e = logits.shape
    chosen = torch.full((t, top), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((t, top), -7.0, device="cuda")
    order = torch.full((t * top,), -7, dtype=torch.int32, device="cuda") if ordered else None
    ends = torch.full((e + 1,), -7, dtype=torch.int32, device="cuda") if ordered else None
    room = torch.full((W.route_experts_workspace_bytes(t, e, top) + 16,), 255, dtype=torch.uint8, device="cuda")
    W.route_experts(logits, chosen, weights, order, ends, bias=None if bias is None else torch.tensor(bias, dtype=torch.float32).cuda(),
                    live=None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda"), workspace=room, **how)
    return [None if x is None else x.cpu().numpy() for x in (chosen, weights, order, ends)]


def check(values, got, top, bias=None, live=None, score=W.SCORE_SOFTMAX, groups=1, top_groups=1, group_best=1, normalise=True,
          scale=1.0):
    chosen, weights, order, ends = got
    t, e = values.shape
    s = decoder8.scores(values, score == W.SCORE_SIGMOID)
    bias = None if bias is None else np.asarray(bias, np.float32)
    for i in range(t):
        if live is not None and i >= live:
            assert (chosen[i] == -1).all() and (weights[i] == 0).all()
            continue
        want = decoder8.route_row(s[i], bias, top, groups, top_groups, group_best)
        assert list(chosen[i]) == want, (i, list(chosen[i]), want)
        w = decoder8.weights(s[i], want, normalise, float(np.float32(scale)))
        assert np.array_equal(np.isnan(weights[i]), np.isnan(w)), i
        ok = np.abs(weights[i] - w) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(w) + 2.0 ** -150
        assert (ok | np.isnan(w)).all(), (i, weights[i], w)
    if order is not None:
        want, begin = decoder8.order(chosen, e)
        assert list(ends) == list(begin)
        assert (order[:len(want)] == want).all() and (order[len(want):] == -7).all()


def logits_of(torch, rng, t, e, name, spread=2.0):
    kind = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]
    x = torch.from_numpy(rng.normal(0, spread, (t, e)).astype(np.float32)).to(kind).cuda()
    return x, x.double().cpu().numpy()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("score", [W.SCORE_SOFTMAX, W.SCORE_SIGMOID])
@pytest.mark.parametrize("t,e,top", [(1, 1, 1), (1, 4, 2), (3, 5, 5), (7, 60, 6), (32, 64, 4), (33, 65, 8), (5, 128, 8), (260, 100, 3),
                                     (9, 256, 32), (70, 257, 1), (2, 513, 9), (6, 1024, 32), (700, 16, 4)])
def test_route(t, e, top, score, name):
    torch = torch_dev()
    rng = np.random.default_rng(t * 31 + e + top)
    logits, values = logits_of(torch, rng, t, e, name)
    how = dict(score=score, normalise=(t + e) % 2 == 0, scale=2.5)
    check(values, run(torch, logits, top, **how), top, **how)


@pytest.mark.parametrize("t", [2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("e,top", [(60, 6), (128, 3), (250, 8), (400, 2), (1000, 5)])
def test_numbers_of_tokens(t, e, top):
    """One block or several, with and without their sums in a launch of their own, a last block that is not full, padding."""
    torch = torch_dev()
    rng = np.random.default_rng(t * 31 + e + top)
    logits, values = logits_of(torch, rng, t, e, "fp16")
    live = t - t // 5
    got = run(torch, logits, top, live=live)
    check(values, got, top, live=live)
    alone = run(torch, logits, top, live=live, ordered=False)
    assert (alone[0] == got[0]).all() and (alone[1] == got[1]).all()


@pytest.mark.parametrize("score", [W.SCORE_SOFTMAX, W.SCORE_SIGMOID])
@pytest.mark.parametrize("t,groups,size,top_groups,best,top", [(50, 8, 32, 4, 2, 8), (20, 2, 2, 1, 2, 2), (9, 64, 2, 5, 2, 7),
                                                               (17, 8, 60, 3, 1, 8), (13, 3, 7, 2, 2, 14), (5, 64, 16, 63, 1, 32),
                                                               (30, 16, 5, 1, 1, 5), (11, 4, 1, 2, 1, 2), (8, 4, 4, 4, 2, 6),
                                                               (130, 16, 64, 7, 2, 32), (64, 5, 100, 2, 2, 16), (65, 3, 33, 1, 1, 33 - 1)])
def test_groups_and_bias(t, groups, size, top_groups, best, top, score):
    torch = torch_dev()
    rng = np.random.default_rng(t + groups * size)
    logits, values = logits_of(torch, rng, t, groups * size, "fp32")
    bias = rng.normal(0, 0.1, groups * size).astype(np.float32)
    how = dict(score=score, groups=groups, top_groups=top_groups, group_best=best)
    check(values, run(torch, logits, top, bias=bias, **how), top, bias=bias, **how)


@pytest.mark.parametrize("e,groups,top_groups", [(8, 1, 1), (70, 1, 1), (64, 8, 3), (300, 4, 2)])
def test_ties_go_to_the_lowest(e, groups, top_groups):
    """Few different values, all values equal, and a bias that makes unequal scores equal."""
    torch = torch_dev()
    rng = np.random.default_rng(e)
    values = rng.integers(0, 3, (40, e)).astype(np.float32)
    values[0] = 1.0
    values[1] = -0.0
    values[2] = np.where(rng.random(e) < 0.5, 0.0, -0.0)
    how = dict(score=W.SCORE_SIGMOID, groups=groups, top_groups=top_groups, group_best=2)
    got = run(torch, torch.from_numpy(values).cuda(), 6, **how)
    check(values, got, 6, **how)
    if top_groups == groups:
        assert list(got[0][0]) == list(range(6)) and list(got[0][1]) == list(range(6))


@pytest.mark.parametrize("score", [W.SCORE_SOFTMAX, W.SCORE_SIGMOID])
@pytest.mark.parametrize("groups", [1, 4])
def test_masked_infinite_and_not_numbers(score, groups):
    """Logits of the type's lowest value, infinities, NaN, rows of nothing else; biases that switch experts off."""
    torch = torch_dev()
    rng = np.random.default_rng(8)
    values = rng.normal(0, 2, (24, 40)).astype(np.float32)
    low = np.finfo(np.float32).min
    values[0, ::2] = low
    values[1] = low
    values[2, :38] = -np.inf
    values[3] = -np.inf
    values[4, 5] = np.inf
    values[5] = np.inf
    values[6, 7] = np.nan
    values[7] = np.nan
    values[8, 1:] = np.nan
    values[9] = np.linspace(-1e30, 1e30, 40)
    values[10] = np.linspace(-800, 800, 40)
    values[11, ::3] = 60.0
    for bias in (None, np.where(np.arange(40) % 3 == 0, -np.inf, 0.0), np.full(40, -np.inf), np.where(np.arange(40) == 3, np.nan, 0.1),
                 np.where(np.arange(40) == 3, np.inf, -np.inf)):
        for normalise in (True, False):
            how = dict(score=score, groups=groups, top_groups=max(1, groups // 2), group_best=2, normalise=normalise)
            check(values, run(torch, torch.from_numpy(values).cuda(), 5, bias=bias, **how), 5, bias=bias, **how)


@pytest.mark.parametrize("live", [-3, 0, 1, 4, 5, 90])
def test_padding(live):
    torch = torch_dev()
    rng = np.random.default_rng(live + 10)
    logits, values = logits_of(torch, rng, 5, 30, "bf16")
    check(values, run(torch, logits, 4, live=live), 4, live=live)


@pytest.mark.parametrize("t,e,top,live", [(4096, 64, 8, None), (16384, 256, 8, None), (6001, 1000, 3, 5000), (300, 4, 4, 17),
                                          (20000, 8, 2, None), (1025, 512, 2, None)])
def test_orders_of_many_routes(t, e, top, live):
    """Order and ends against a stable sort of the choice; a hundred rows' choice against the oracle."""
    torch = torch_dev()
    rng = np.random.default_rng(t)
    logits, values = logits_of(torch, rng, t, e, "fp32")
    logits[:, e // 2] += 3
    values[:, e // 2] = logits[:, e // 2].double().cpu().numpy()
    got = run(torch, logits, top, live=live)
    again = run(torch, logits, top, live=live)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))
    flat = got[0].reshape(-1)
    there = np.flatnonzero(flat >= 0)
    want = there[np.argsort(flat[there], kind="stable")]
    assert (got[2][:len(want)] == want).all() and (got[2][len(want):] == -7).all()
    assert (got[3] == np.concatenate([[0], np.cumsum(np.bincount(flat[there], minlength=e))])).all()
    rows = np.sort(rng.permutation(t if live is None else live)[:100])
    check(values[rows], [got[0][rows], got[1][rows], None, None], top)


def test_strides_streams_and_neighbours():
    torch = torch_dev()
    rng = np.random.default_rng(6)
    wide, values = logits_of(torch, rng, 11, 100, "fp16")
    logits = wide[:, 33:33 + 50]                                # two bytes past a multiple of four
    memory = torch.full((200,), -9, dtype=torch.int32, device="cuda")
    weights = torch.full((200,), -9.0, device="cuda")
    chosen, w = memory[3:3 + 33].view(11, 3), weights[5:5 + 33].view(11, 3)
    order, ends = memory[50:83], memory[90:141]
    room = torch.empty(W.route_experts_workspace_bytes(11, 50, 3), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    W.route_experts(logits, chosen, w, order, ends, workspace=room, stream=side)
    side.synchronize()
    check(values[:, 33:83], [x.cpu().numpy() for x in (chosen, w, order, ends)], 3)
    for a, b in ((0, 3), (36, 50), (83, 90), (141, 200)):
        assert (memory[a:b] == -9).all()
    assert (weights[:5] == -9).all() and (weights[38:] == -9).all()


def test_without_order_and_empty():
    torch = torch_dev()
    rng = np.random.default_rng(7)
    logits, values = logits_of(torch, rng, 10, 20, "fp32")
    check(values, run(torch, logits, 2, ordered=False), 2)
    ends = torch.full((21,), 5, dtype=torch.int32, device="cuda")
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    W.route_experts(logits[:0], none, none.float(), none[:, 0].contiguous(), ends)
    assert (ends == 0).all()


def test_refused():
    torch = torch_dev()
    logits = torch.zeros((4, 8), device="cuda")
    chosen, w = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    order, ends = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    room = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    for bad in ((logits.double(), chosen, w), (logits, chosen.long(), w), (logits, chosen[:3], w), (logits, chosen, w[:, :1]),
                (logits.t(), chosen, w), (logits, chosen, w, order, None), (logits, chosen, w, order[:7], ends),
                (logits, chosen, w, order, ends[:8])):
        with pytest.raises(ValueError):
            W.route_experts(*bad, workspace=room)
    for kw in (dict(groups=3), dict(score=2), dict(groups=8, top_groups=1), dict(scale=float("nan"))):
        with pytest.raises(W.WinoError):
            W.route_experts(logits, chosen, w, order, ends, workspace=room, **kw)
    many = torch.zeros((65, 8), device="cuda")                  # more than one block: the order needs room
    with pytest.raises(W.WinoError):
        W.route_experts(many, torch.zeros((65, 2), dtype=torch.int32, device="cuda"), torch.zeros((65, 2), device="cuda"),
                        torch.zeros(130, dtype=torch.int32, device="cuda"), ends)
    with pytest.raises(ValueError):
        W.route_experts(logits, chosen, w, bias=logits[0].half())

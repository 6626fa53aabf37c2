"""w8_experts_matmul against float64 products of the same codes (bounds as for
w8_matmul), and the 8-bit operators together as a layer of experts runs them.

A weighted sum adds `top` products, each off by 3 2^-24 of itself, in fp32: a
rounding of each product with its weight and one for each addition."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder8

from decoder_util import ROUND, TINY, dtype, half, host
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def layer(torch, rng, t, e, top, n, k, shared, skew=0.0):
    """x, its scales, weights, their scales, chosen, order, ends."""
    rows = t if shared else t * top
    x = torch.from_numpy(rng.integers(-127, 128, (rows, k), dtype=np.int8)).cuda()
    w = torch.from_numpy(rng.integers(-127, 128, (e, n, k), dtype=np.int8)).cuda()
    xs = torch.from_numpy(rng.uniform(0.5, 2, rows).astype(np.float32) * 0.01).cuda()
    ws = torch.from_numpy(rng.uniform(0.5, 2, (e, n)).astype(np.float32) * 0.01).cuda()
    liked = rng.normal(0, 1, (t, e)) + skew * rng.normal(0, 1, e)
    chosen = np.argsort(-liked, -1)[:, :top].astype(np.int32)
    return x, xs, w, ws, chosen


def grouped(torch, chosen, e):
    routes, ends = decoder8.order(chosen, e)
    order = np.full(chosen.size, -5, np.int32)
    order[:len(routes)] = routes
    return torch.from_numpy(order).cuda(), torch.from_numpy(ends.astype(np.int32)).cuda(), routes, ends


def products(x, xs, w, ws, routes, ends, total):
    """float64 on the GPU, NaN where a route is not in the order."""
    torch = torch_dev()
    y = torch.full((total, w.shape[1]), float("nan"), dtype=torch.float64, device="cuda")
    share = total // len(x)
    for e in range(len(w)):
        if ends[e] < ends[e + 1]:
            r = torch.from_numpy(np.asarray(routes[ends[e]:ends[e + 1]])).cuda()
            sums = x[r // share].double() @ w[e].double().t()
            y[r] = sums * xs[r // share].double()[:, None] * ws[e].double()
    return y


def close(y, ref, size, roundings, name):
    err = 2.0 ** -24 * (roundings + 0.01) * size
    bound = err + ROUND[name] * (ref.abs() + err) + TINY[name]
    bad = ~((y.double() - ref).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


SIZES = [(1, 1, 1, 1, 16), (1, 8, 2, 100, 64), (3, 5, 5, 33, 272), (7, 60, 6, 48, 144), (32, 64, 6, 130, 2064), (40, 4, 2, 257, 96),
         (200, 3, 1, 40, 512), (150, 8, 4, 129, 1040), (600, 16, 8, 72, 208), (333, 128, 8, 20, 64), (64, 1024, 2, 17, 32),
         (3, 2, 1, 4096, 4096), (1000, 2, 2, 300, 128), (2100, 6, 3, 260, 48),
         (186, 4, 2, 1519, 7104), (78, 16, 2, 562, 4528), (1343, 4, 2, 367, 7568),
         (1, 256, 8, 130, 272), (3, 1024, 4, 70, 144), (2, 65, 3, 257, 2064)]


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("t,e,top,n,k", SIZES)
def test_products(t, e, top, n, k, shared, name):
    torch = torch_dev()
    rng = np.random.default_rng(t * 31 + e * 7 + n + k)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, top, n, k, shared, skew=1.0 if t % 2 else 0.0)
    order, ends, routes, begin = grouped(torch, chosen, e)
    ref = products(x, xs, w, ws, routes, begin, t * top)
    y = torch.full((t * top, n), float("nan"), dtype=dtype(torch, name), device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, y)
    close(y, ref, ref.abs(), 3, name)
    weights = torch.from_numpy(rng.uniform(0, 1, (t, top)).astype(np.float32)).cuda()
    room = torch.full((W.w8_experts_matmul_workspace_bytes(t * top, n, True),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((t, n), float("nan"), dtype=dtype(torch, name), device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, out, chosen=torch.from_numpy(chosen).cuda(), weights=weights, workspace=room)
    parts = ref.view(t, top, n) * weights.double()[..., None]
    close(out, parts.sum(1), parts.abs().sum(1), 4 + top, name)


def test_against_the_oracle():
    torch = torch_dev()
    rng = np.random.default_rng(3)
    x, xs, w, ws, chosen = layer(torch, rng, 9, 4, 2, 21, 48, True)
    order, ends, routes, begin = grouped(torch, chosen, 4)
    y = torch.empty((18, 21), dtype=torch.float16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, y)
    ref = decoder8.experts_product(*(t.cpu().numpy() for t in (x, xs, w, ws)), routes, begin, 18)
    err = 2.0 ** -24 * 3.01 * np.abs(ref)
    assert (np.abs(host(y) - ref) <= err + ROUND["fp16"] * (np.abs(ref) + err) + TINY["fp16"]).all()


@pytest.mark.parametrize("t,e,top,n,k", [(2100, 2, 2, 2052, 8208), (2100, 2, 1, 2050, 6160), (4500, 3, 2, 1000, 6160),
                                         (4100, 70, 2, 600, 6160), (9000, 2, 1, 4100, 528)])
def test_more_tiles_than_compute_units(t, e, top, n, k):
    """Workgroups that go on from tile to tile, and last tiles in parts of k, with routes that are nobody's."""
    torch = torch_dev()
    rng = np.random.default_rng(t + n + k)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, top, n, k, True, skew=0.5)
    chosen[rng.integers(0, t, 50)] = -1
    order, ends, routes, begin = grouped(torch, chosen, e)
    ref = products(x, xs, w, ws, routes, begin, t * top)
    there = torch.from_numpy((chosen >= 0).reshape(-1)).cuda()
    chosen = torch.from_numpy(chosen).cuda()
    weights = torch.from_numpy(rng.uniform(0, 1, (t, top)).astype(np.float32)).cuda()
    parts = torch.where(there[:, None], ref, 0.0).view(t, top, n) * weights.double()[..., None]
    products_bytes = t * top * n * 4
    first = None
    for more in (True, False):
        need = W.w8_experts_matmul_workspace_bytes(t * top, n, False)
        room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda") if more else None
        y = torch.full((t * top + 1, n), 77.0, dtype=torch.bfloat16, device="cuda")
        W.w8_experts_matmul(x, xs, w, ws, order, ends, y[:-1], workspace=room)
        close(y[:-1][there], ref[there], ref[there].abs(), 3, "bf16")
        assert (y[:-1][~there] == 77).all() and (y[-1] == 77).all()
        assert room is None or (room[need:] == 255).all()
        need = W.w8_experts_matmul_workspace_bytes(t * top, n, True) if more else products_bytes
        room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((t + 1, n), 77.0, dtype=torch.bfloat16, device="cuda")
        W.w8_experts_matmul(x, xs, w, ws, order, ends, out[:-1], chosen=chosen, weights=weights, workspace=room[:need])
        close(out[:-1], parts.sum(1), parts.abs().sum(1), 4 + top, "bf16")
        assert (out[-1] == 77).all() and (room[need:] == 255).all()
        if first is None:
            first = y, out
        assert torch.equal(first[0], y) and torch.equal(first[1], out), "another workspace gives another result"


@pytest.mark.parametrize("t,e", [(5, 3), (90, 2), (400, 5), (4, 300), (30, 1000)])
def test_missing_routes(t, e):
    """Padding tokens, single routes without an expert, and experts without routes."""
    torch = torch_dev()
    rng = np.random.default_rng(t)
    top, n, k = 2, 45, 80
    x, xs, w, ws, chosen = layer(torch, rng, t, e, top, n, k, True)
    chosen[chosen == e - 1] = -1
    chosen[t - 2:] = -1
    order, ends, routes, begin = grouped(torch, chosen, e)
    ref = products(x, xs, w, ws, routes, begin, t * top)
    there = torch.from_numpy((chosen >= 0).reshape(-1)).cuda()
    y = torch.full((t * top, n), 77.0, dtype=torch.bfloat16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, y)
    close(y[there], ref[there], ref[there].abs(), 3, "bf16")
    assert (y[~there] == 77).all()
    weights = torch.from_numpy(rng.uniform(0, 1, (t, top)).astype(np.float32)).cuda()
    weights[t - 1] = float("nan")                               # of a token without routes
    room = torch.full((W.w8_experts_matmul_workspace_bytes(t * top, n, True),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((t, n), 77.0, dtype=torch.bfloat16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, out, chosen=torch.from_numpy(chosen).cuda(), weights=weights, workspace=room)
    parts = torch.where(there.view(t, top, 1), ref.view(t, top, n) * weights.double()[..., None], 0.0)
    close(out, parts.sum(1), parts.abs().sum(1), 4 + top, "bf16")
    assert (out[t - 2:] == 0).all()


@pytest.mark.parametrize("t", [6, 300])
def test_orders_out_of_range(t):
    """Routes below 0 or past the last are left out, ends are cut to the order: nothing outside is read or written."""
    torch = torch_dev()
    rng = np.random.default_rng(t)
    x, xs, w, ws, chosen = layer(torch, rng, t, 3, 1, 20, 64, True)
    order, ends, routes, begin = grouped(torch, chosen, 3)
    ref = products(x, xs, w, ws, routes, begin, t)
    bad = order.clone()
    bad[1], bad[3] = -1, t
    bad[4] = 2 ** 31 - 1
    memory = torch.full((t + 2, 20), 77.0, dtype=torch.float16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, bad, ends, memory[1:t + 1])
    gone = order[[1, 3, 4]].long()
    kept = torch.ones(t, dtype=torch.bool, device="cuda")
    kept[gone] = False
    y = memory[1:t + 1]
    close(y[kept], ref[kept], ref[kept].abs(), 3, "fp16")
    assert (y[gone] == 77).all() and (memory[0] == 77).all() and (memory[t + 1] == 77).all()
    for wrong in ([-5, 2, 1, 10 ** 9], [0, 10 ** 9, 10 ** 9, 10 ** 9], [5, 4, 3, 2]):
        memory.fill_(77.0)
        W.w8_experts_matmul(x, xs, w, ws, order, torch.tensor(wrong, dtype=torch.int32, device="cuda"), memory[1:t + 1])
        assert (memory[0] == 77).all() and (memory[t + 1] == 77).all()


@pytest.mark.parametrize("t,e,n,k", [(40, 9, 70, 96), (700, 70, 130, 64), (4200, 5, 1000, 6160), (4200, 2, 2052, 8208)])
def test_ends_that_go_back(t, e, n, k):
    """Every other expert claims all routes: more tiles than routes can have, in the lists of the XCDs and in the parts of the
    last ones.  Nothing outside is read or written."""
    torch = torch_dev()
    rng = np.random.default_rng(t + n)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, 1, n, k, True)
    order, ends, routes, begin = grouped(torch, chosen, e)
    bad = torch.tensor([0, t] * (e // 2 + 1), dtype=torch.int32, device="cuda")[:e + 1].contiguous()
    need = W.w8_experts_matmul_workspace_bytes(t, n, False)
    room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    memory = torch.full((t + 2, n), 77.0, dtype=torch.float16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, bad, memory[1:t + 1], workspace=room[:need])
    assert (memory[0] == 77).all() and (memory[t + 1] == 77).all() and (room[need:] == 255).all()
    W.w8_experts_matmul(x, xs, w, ws, order, ends, memory[1:t + 1], workspace=room[:need])
    ref = products(x, xs, w, ws, routes, begin, t)
    close(memory[1:t + 1], ref, ref.abs(), 3, "fp16")


@pytest.mark.parametrize("t", [8, 500])
def test_strided_rows_and_neighbours(t):
    torch = torch_dev()
    rng = np.random.default_rng(t)
    n, k = 50, 96
    x, xs, w, ws, chosen = layer(torch, rng, t, 4, 2, n, k + 32, False)
    w = w[:, :, :k].contiguous()
    order, ends, routes, begin = grouped(torch, chosen, 4)
    ref = products(x[:, 16:16 + k], xs, w, ws, routes, begin, 2 * t)
    wide = torch.full((2 * t + 2, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    W.w8_experts_matmul(x[:, 16:16 + k], xs, w, ws, order, ends, wide[1:2 * t + 1, 3:3 + n])
    close(wide[1:2 * t + 1, 3:3 + n], ref, ref.abs(), 3, "bf16")
    assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :3] == 7).all() and (wide[:, 3 + n:] == 7).all()


def test_empty_and_refused():
    torch = torch_dev()
    rng = np.random.default_rng(1)
    x, xs, w, ws, chosen = layer(torch, rng, 4, 3, 2, 8, 32, True)
    order, ends, *_ = grouped(torch, chosen, 3)
    y = torch.zeros((8, 8), dtype=torch.bfloat16, device="cuda")
    ch, gw = torch.from_numpy(chosen).cuda(), torch.ones((4, 2), device="cuda")
    W.w8_experts_matmul(x[:0], xs[:0], w, ws, order[:0], ends * 0, y[:0])
    W.w8_experts_matmul(x, xs, w[:, :0], ws[:, :0], order, ends, y[:, :0])
    for bad in ((x[:3], xs[:3], w, ws, order, ends, y), (x, xs[:3], w, ws, order, ends, y), (x, xs, w[0], ws, order, ends, y),
                (x, xs, w, ws[:2], order, ends, y), (x, xs, w, ws, order[:7], ends, y), (x, xs, w, ws, order, ends[:3], y),
                (x, xs, w, ws, order, ends, y[:4]), (x, xs, w, ws, order.long(), ends, y), (x, xs, w, ws, order, ends, y.float()),
                (x, xs, w, ws, order, ends, y, ch, None), (x, xs, w, ws, order, ends, y, None, gw),
                (x, xs, w, ws, order, ends, y, ch, gw), (x, xs, w, ws, order, ends, y[:4], ch[:3], gw),
                (x, xs, w, ws, order, ends, y[:4], ch, gw[:3])):
        with pytest.raises(ValueError):
            W.w8_experts_matmul(*bad)
    with pytest.raises(W.WinoError):
        W.w8_experts_matmul(x, xs, w, ws, order, ends, y[:4], ch, gw)      # no workspace


class Layer:
    """A layer of experts on the 8-bit operators: router, first products, silu(gate) * up, products back."""

    def __init__(self, torch, rng, hidden, inner, experts, top, most):
        def codes(*shape):
            w = torch.from_numpy(rng.normal(0, shape[-1] ** -0.5, shape).astype(np.float32)).to(torch.bfloat16).cuda()
            c, s = torch.empty(shape, dtype=torch.int8, device="cuda"), torch.empty(shape[:-1], device="cuda")
            W.w8_quantize(w.view(-1, shape[-1]), c.view(-1, shape[-1]), s.view(-1))
            return c, s
        self.torch, self.top, self.experts, self.inner = torch, top, experts, inner
        self.router, self.up, self.down = codes(experts, hidden), codes(experts, 2 * inner, hidden), codes(experts, hidden, inner)
        self.head = codes(300, hidden)
        need = max(W.route_experts_workspace_bytes(most, experts, top), W.w8_experts_matmul_workspace_bytes(most * top, hidden, True),
                   W.w8_matmul_workspace_bytes(most, 300, hidden), W.w8_matmul_workspace_bytes(most, experts, hidden))
        self.room = torch.empty(need + 16, dtype=torch.uint8, device="cuda")

    def quantize(self, x):
        codes = self.torch.empty(x.shape, dtype=self.torch.int8, device="cuda")
        scales = self.torch.empty(len(x), device="cuda")
        W.w8_quantize(x, codes, scales)
        return codes, scales

    def __call__(self, x, live=None):
        """Everything that the step works out, by name."""
        torch, (t, hidden) = self.torch, x.shape
        empty = lambda *shape: torch.empty(shape, dtype=x.dtype, device="cuda")     # noqa: E731
        ints = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        codes, scales = self.quantize(x)
        logits, h, y, out = empty(t, self.experts), empty(t * self.top, 2 * self.inner), empty(t, hidden), empty(t, 300)
        W.w8_matmul(codes, scales, *self.router, logits, workspace=self.room)
        chosen, order, ends = ints(t, self.top), ints(t * self.top), ints(self.experts + 1)
        weights = torch.empty((t, self.top), device="cuda")
        W.route_experts(logits, chosen, weights, order, ends, live=live, workspace=self.room)
        h.zero_()
        W.w8_experts_matmul(codes, scales, *self.up, order, ends, h)
        gate, up = h.chunk(2, -1)
        inside = torch.nn.functional.silu(gate) * up
        icodes, iscales = self.quantize(inside)
        W.w8_experts_matmul(icodes, iscales, *self.down, order, ends, y, chosen=chosen, weights=weights, workspace=self.room)
        ycodes, yscales = self.quantize(y)
        W.w8_matmul(ycodes, yscales, *self.head, out, workspace=self.room)
        return dict(codes=codes, scales=scales, logits=logits, chosen=chosen, weights=weights, order=order, ends=ends, h=h,
                    inside=inside, icodes=icodes, iscales=iscales, y=y, ycodes=ycodes, yscales=yscales, out=out)


@pytest.mark.parametrize("t", [1, 5, 64, 300])
def test_a_layer_of_experts(t):
    """Each operator of the run against its formula on the operands that the run handed to it."""
    torch = torch_dev()
    rng = np.random.default_rng(t)
    net = Layer(torch, rng, 256, 80, 12, 3, t)
    x, xv = half(torch, rng.normal(0, 1, (t, 256)), "bf16")
    r = {k: v.cpu() for k, v in net(x).items()}
    for src, codes, scales in ((xv, "codes", "scales"), (host(r["inside"]), "icodes", "iscales"), (host(r["y"]), "ycodes", "yscales")):
        for i in range(0, len(src), max(1, len(src) // 7)):
            want, scale = decoder8.quantize_row(src[i])
            assert (r[codes][i].numpy() == want).all() and float(r[scales][i]) == np.float32(float(scale))

    def product(x, xs, w):
        return decoder8.product(r[x].numpy(), r[xs].numpy(), *(v.cpu().numpy() for v in w))
    for got, ref in ((r["logits"], product("codes", "scales", net.router)), (r["out"], product("ycodes", "yscales", net.head))):
        close(got, torch.from_numpy(ref), torch.from_numpy(np.abs(ref)), 3, "bf16")
    s = decoder8.scores(host(r["logits"]), False)
    for i in range(t):
        want = decoder8.route_row(s[i], None, 3, 1, 1, 1)
        assert list(r["chosen"][i]) == want
        assert np.allclose(r["weights"][i].numpy(), decoder8.weights(s[i], want, True, 1.0), rtol=2.0 ** -23, atol=0)
    routes, ends = decoder8.order(r["chosen"].numpy(), 12)
    assert (r["order"].numpy() == routes).all() and (r["ends"].numpy() == ends).all()
    up, down = ([v.cpu().numpy() for v in w] for w in (net.up, net.down))
    ref = torch.from_numpy(decoder8.experts_product(r["codes"].numpy(), r["scales"].numpy(), *up, routes, ends, 3 * t))
    close(r["h"], ref, ref.abs(), 3, "bf16")
    ref = torch.from_numpy(decoder8.experts_product(r["icodes"].numpy(), r["iscales"].numpy(), *down, routes, ends, 3 * t))
    ref = ref.view(t, 3, 256) * r["weights"].double()[..., None]
    close(r["y"], ref.sum(1), ref.abs().sum(1), 7, "bf16")


def test_captured_layers_of_a_padded_batch():
    """Two graphs that share their workspace, replayed several times with other inputs, other lengths and eager calls in
    between: what they give is what the eager calls give, and padding changes nothing for the tokens before it."""
    torch = torch_dev()
    rng = np.random.default_rng(11)
    most = 40
    net = Layer(torch, rng, 128, 48, 16, 4, most)
    x = torch.zeros((most, 128), dtype=torch.bfloat16, device="cuda")
    live = torch.tensor([most], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net(x, live)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for rows in (most, 7):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = net(x[:rows], live)
        graphs.append((g, rows, got))
    for step in range(5):
        data = half(torch, rng.normal(0, 1, (most, 128)), "bf16")[0]
        n = int(rng.integers(0, most + 1))
        x.copy_(data)
        live.fill_(n)
        for g, rows, got in graphs:
            g.replay()
            torch.cuda.synchronize()
            result = {k: v.clone() for k, v in got.items()}
            want = net(data[:rows], live)
            used = min(n, rows)
            assert int(result["ends"][-1]) == 4 * used
            for k in ("codes", "logits", "chosen", "weights", "ends", "h", "y", "out"):
                assert torch.equal(result[k], want[k]), (step, rows, k)
            assert torch.equal(result["order"][:4 * used], want["order"][:4 * used])
            if used:
                alone = net(data[:used])
                assert torch.equal(alone["y"], result["y"][:used])
            assert (result["y"][used:] == 0).all()

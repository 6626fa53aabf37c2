"""Every kernel of the 8-bit decoder operators on sizes that take it
(decoder8_sizes.py), against float64; bounds as in the operators' own tests."""
import numpy as np
import pytest

import decoder8_sizes as sizes
import paper_2209_12982_amd as W
from oracle import decoder8

from decoder_util import dtype, half
from gpu_util import torch_dev
from test_gpu_route_experts import check as check_routes
from test_gpu_route_experts import logits_of, run
from test_gpu_w8_experts import close, grouped, layer, products
from test_gpu_w8_matmul import check, operands

pytestmark = pytest.mark.gpu


def cases(table):
    return [pytest.param(s, id=f"{'-'.join(filter(None, key)).replace(' ', '_')}-{'x'.join(map(str, s))}")
            for key, many in table.items() for s in many]


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("size", cases(sizes.MATMUL))
def test_matmul(size, name):
    """With a workspace and without one, rows of y at 16 bytes and past it, nothing beside y written."""
    torch = torch_dev()
    m, n, k = size
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    x, xs, w, ws = operands(torch, rng, m, n, k, low=-128)
    xs *= (1024 / k) ** 0.5
    bias = half(torch, rng.normal(0, 1, n), name)[0] if n % 2 else None
    need = W.w8_matmul_workspace_bytes(m, n, k)
    room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    wide = torch.empty((m + 2, n + 16), dtype=dtype(torch, name), device="cuda")
    first = None
    for left, space in ((8, room[:need]), (7, None)):
        wide.fill_(7.0)
        y = wide[1:m + 1, left:left + n]
        y.fill_(float("nan"))
        W.w8_matmul(x, xs, w, ws, y, bias=bias, workspace=space)
        if first is None:
            check(y, x, xs, w, ws, bias, name)
            first = y.clone()
        assert torch.equal(first, y), "another workspace gives another result"
        assert (wide[0] == 7).all() and (wide[m + 1] == 7).all() and (wide[:, :left] == 7).all() and (wide[:, left + n:] == 7).all()
    assert (room[need:] == 255).all()


@pytest.mark.parametrize("m,n,k,apart", sizes.MATMUL_FAR + sizes.MATMUL_NEAR)
def test_matmul_of_far_rows(m, n, k, apart):
    """Rows of x further apart in a tile than 32 bits hold, and just less."""
    torch = torch_dev()
    rng = np.random.default_rng(m + n + k)
    x, xs, w, ws = operands(torch, rng, m, n, k)
    xs *= (1024 / k) ** 0.5
    far = torch.empty((m, apart), dtype=torch.int8, device="cuda")
    far[:, :k] = x
    y = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    W.w8_matmul(far[:, :k], xs, w, ws, y)
    check(y, x, xs, w, ws, None, "bf16")


def check_experts(torch, rng, x, far, xs, w, ws, chosen, top, name):
    """Products and weighted sums with all workspaces; x: the rows that `far` holds too."""
    e, n, t = w.shape[0], w.shape[1], len(chosen)
    order, ends, routes, begin = grouped(torch, chosen, e)
    ref = products(x, xs, w, ws, routes, begin, t * top)
    there = torch.from_numpy((chosen >= 0).reshape(-1)).cuda()
    chosen = torch.from_numpy(chosen).cuda()
    weights = torch.from_numpy(rng.uniform(0, 1, (t, top)).astype(np.float32)).cuda()
    parts = torch.where(there[:, None], ref, 0.0).view(t, top, n) * weights.double()[..., None]
    first = None
    for more in (True, False):
        need = W.w8_experts_matmul_workspace_bytes(t * top, n, False)
        room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        y = torch.full((t * top + 1, n), 77.0, dtype=dtype(torch, name), device="cuda")
        W.w8_experts_matmul(far, xs, w, ws, order, ends, y[:-1], workspace=room[:need] if more else None)
        assert (y[:-1][~there] == 77).all() and (y[-1] == 77).all() and (room[need:] == 255).all()
        need = W.w8_experts_matmul_workspace_bytes(t * top, n, True) if more else t * top * n * 4
        room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((t + 1, n), 77.0, dtype=dtype(torch, name), device="cuda")
        W.w8_experts_matmul(far, xs, w, ws, order, ends, out[:-1], chosen=chosen, weights=weights, workspace=room[:need])
        assert (out[-1] == 77).all() and (room[need:] == 255).all()
        if first is None:
            close(y[:-1][there], ref[there], ref[there].abs(), 3, name)
            close(out[:-1], parts.sum(1), parts.abs().sum(1), 4 + top, name)
            first = y, out
        assert torch.equal(first[0], y) and torch.equal(first[1], out), "another workspace gives another result"


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("size", cases(sizes.EXPERTS))
def test_experts(size, name):
    """Routes of uneven experts, some of them nobody's."""
    torch = torch_dev()
    t, e, top, n, k = size
    rng = np.random.default_rng(t * 31 + e * 7 + n + k)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, top, n, k, True, skew=0.5)
    xs *= (256 / k) ** 0.5
    chosen[rng.integers(0, t, t // 8)] = -1
    check_experts(torch, rng, x, x, xs, w, ws, chosen, top, name)


@pytest.mark.parametrize("t,e,n,k", [(900, 64, 200, 272), (500, 512, 1000, 144), (37, 8, 33, 2064), (3000, 16, 257, 528), (5000, 4, 300, 1040)])
def test_one_expert_has_all_routes(t, e, n, k):
    """As uneven as routes can be: sets of rows one after the other, the most tiles that one expert can have, and none for others."""
    torch = torch_dev()
    rng = np.random.default_rng(t + e)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, 1, n, k, True)
    chosen[:] = e - 2
    check_experts(torch, rng, x, x, xs, w, ws, chosen, 1, "bf16")


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("t,e,top,n,k,apart", sizes.EXPERTS_FAR + sizes.EXPERTS_NEAR)
def test_experts_of_far_rows(t, e, top, n, k, apart, shared):
    """Rows of x past 2^32 bytes, and past 2^31, for each token and for each route."""
    torch = torch_dev()
    rng = np.random.default_rng(t + n)
    x, xs, w, ws, chosen = layer(torch, rng, t, e, top, n, k, shared)
    far = torch.empty((len(x), apart), dtype=torch.int8, device="cuda")
    far[:, :k] = x
    chosen[t // 2] = -1
    check_experts(torch, rng, x, far[:, :k], xs, w, ws, chosen, top, "fp16")


@pytest.mark.parametrize("name", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("size", cases(sizes.ROUTE))
def test_route(size, name):
    """The choice of some tokens against the oracle, the order against a stable sort of the choice."""
    torch = torch_dev()
    t, e, top = size
    rng = np.random.default_rng(t * 31 + e + top)
    logits, values = logits_of(torch, rng, t, e, name)
    live = t - t // 9
    got = run(torch, logits, top, live=live)
    flat = got[0].reshape(-1)
    there = np.flatnonzero(flat >= 0)
    assert len(there) == live * top and (got[0][live:] == -1).all() and (got[1][live:] == 0).all()
    want = there[np.argsort(flat[there], kind="stable")]
    assert (got[2][:len(want)] == want).all() and (got[2][len(want):] == -7).all()
    assert (got[3] == np.concatenate([[0], np.cumsum(np.bincount(flat[there], minlength=e))])).all()
    rows = np.sort(rng.permutation(live)[:100])
    check_routes(values[rows], [got[0][rows], got[1][rows], None, None], top)


def ends_of(rows, some=300):
    """The first rows, the last ones, and some between."""
    step = max(1, rows // some)
    return sorted(set(range(min(rows, 70))) | set(range(max(0, rows - 70), rows)) | set(range(0, rows, step)))


@pytest.mark.parametrize("m,n,k", [(1 << 20, 40, 16), (1 << 20, 2100, 16), (3, 1 << 24, 16), (200, 5000000, 32)])
def test_matmul_of_the_most_rows_and_outputs(m, n, k):
    """Up to 2^20 rows, 2^24 outputs and more than 2^31 results."""
    torch = torch_dev()
    gen = torch.Generator("cuda").manual_seed(m + n)
    x, w = (torch.randint(-127, 128, (rows, k), generator=gen, device="cuda", dtype=torch.int8) for rows in (m, n))
    xs, ws = (0.01 + torch.rand(rows, generator=gen, device="cuda") for rows in (m, n))
    y = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    W.w8_matmul(x, xs, w, ws, y)
    assert not torch.isnan(y.view(-1)[::977]).any()
    rows, cols = (torch.tensor(ends_of(size), device="cuda") for size in (m, n))
    check(y[rows][:, cols], x[rows], xs[rows], w[cols], ws[cols], None, "bf16")


@pytest.mark.parametrize("m,k", [((1 << 24) - 1, 16), (3, 1 << 20)])
def test_quantize_the_most_rows(m, k):
    torch = torch_dev()
    gen = torch.Generator("cuda").manual_seed(m)
    x = torch.randn((m, k), generator=gen, device="cuda", dtype=torch.bfloat16)
    codes = torch.full((m, k), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((m,), -1.0, device="cuda")
    W.w8_quantize(x, codes, scales)
    assert (scales > 0).all()
    for i in ends_of(m, 20):
        some = ends_of(k, 2000)
        row = x[i].double().cpu().numpy()
        top = np.argmax(np.abs(row))
        want, scale = decoder8.quantize_row(np.append(row[some], row[top]))
        assert (codes[i].cpu().numpy()[some] == want[:-1]).all() and scales[i] == np.float32(float(scale)), i


@pytest.mark.parametrize("t,e,top", [(1 << 22, 5, 1), (1 << 17, 64, 32), (1 << 19, 1024, 8)])
def test_route_the_most_tokens(t, e, top):
    torch = torch_dev()
    gen = torch.Generator("cuda").manual_seed(t + e)
    logits = torch.randn((t, e), generator=gen, device="cuda", dtype=torch.float32)
    got = run(torch, logits, top)
    flat = got[0].reshape(-1)
    assert flat.min() >= 0 and flat.max() < e
    assert (got[2] == np.argsort(flat, kind="stable")).all()
    assert (got[3] == np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=e))])).all()
    rows = ends_of(t, 50)
    check_routes(logits[rows].double().cpu().numpy(), [got[0][rows], got[1][rows], None, None], top)


@pytest.mark.parametrize("t,e,top,n,k", [(1 << 20, 3, 4, 33, 16), (1 << 21, 2, 2, 520, 16)])
def test_experts_of_the_most_routes(t, e, top, n, k):
    """2^22 routes, and more than 2^31 products."""
    torch = torch_dev()
    gen = torch.Generator("cuda").manual_seed(t + n)
    x = torch.randint(-127, 128, (t, k), generator=gen, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (e, n, k), generator=gen, device="cuda", dtype=torch.int8)
    xs, ws = 0.01 + torch.rand(t, generator=gen, device="cuda"), 0.01 + torch.rand((e, n), generator=gen, device="cuda")
    chosen = torch.randint(0, e, (t, top), generator=gen, device="cuda", dtype=torch.int32)
    flat = chosen.flatten()
    order = torch.sort(flat, stable=True).indices.int()
    ends = torch.cat((torch.zeros(1, device="cuda", dtype=torch.long), torch.bincount(flat, minlength=e).cumsum(0))).int()
    weights = torch.rand((t, top), generator=gen, device="cuda")
    rows = torch.tensor(ends_of(t), device="cuda")
    ref = torch.stack([(x[rows].double()[:, None] * w[chosen[rows, j].long()].double()).sum(-1)
                       * xs[rows].double()[:, None] * ws[chosen[rows, j].long()].double() for j in range(top)], 1)
    y = torch.full((t * top, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, y)
    assert not torch.isnan(y.view(-1)[::977]).any()
    close(y.view(t, top, n)[rows], ref, ref.abs(), 3, "bf16")
    del y
    room = torch.empty(W.w8_experts_matmul_workspace_bytes(t * top, n, True), dtype=torch.uint8, device="cuda")
    out = torch.full((t, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    W.w8_experts_matmul(x, xs, w, ws, order, ends, out, chosen=chosen, weights=weights, workspace=room)
    parts = ref * weights[rows].double()[..., None]
    close(out[rows], parts.sum(1), parts.abs().sum(1), 4 + top, "bf16")

"""w8_matmul against float64 products of the same codes.

The sum of products is exact.  It becomes fp32 (2^-24 of itself), is multiplied
by x_scale (2^-24) and by w_scale with the bias added (2^-24 of the result), and
the result is rounded to 16 bits."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder8

from decoder_util import ROUND, TINY, dtype, half, host
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def operands(torch, rng, m, n, k, low=-127):
    x = torch.from_numpy(rng.integers(low, 128, (m, k), dtype=np.int8)).cuda()
    w = torch.from_numpy(rng.integers(low, 128, (n, k), dtype=np.int8)).cuda()
    xs = torch.from_numpy(rng.uniform(0.5, 2, m).astype(np.float32) * 0.01).cuda()
    ws = torch.from_numpy(rng.uniform(0.5, 2, n).astype(np.float32) * 0.01).cuda()
    return x, xs, w, ws


def check(y, x, xs, w, ws, bias, name):
    torch = torch_dev()
    sums = x.double() @ w.double().t()                          # whole numbers below 2^53: exact
    part = sums * xs.double()[:, None] * ws.double()
    ref = part if bias is None else part + bias.double()
    err = 2.0 ** -24 * (2.01 * part.abs() + 1.01 * ref.abs())
    bound = err + ROUND[name] * (ref.abs() + err) + TINY[name]
    bad = ~((y.double() - ref).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"
    if bias is None:                                            # the same three roundings, bit for bit
        same = ((sums.float() * xs[:, None]) * ws).to(y.dtype)
        assert torch.equal(y, same)


SIZES = [(1, 1, 16), (1, 17, 64), (1, 4096, 4096), (2, 16, 96), (3, 33, 160), (5, 203, 2080), (8, 64, 512), (15, 130, 1024),
         (16, 48, 4096), (17, 100, 544), (33, 31, 256), (48, 129, 1040), (64, 257, 2064), (1, 40, 16384), (31, 64, 131056),
         (65, 7, 48), (70, 20, 128), (100, 300, 1008), (128, 128, 128), (129, 127, 4096), (333, 1003, 2080), (257, 520, 144),
         (300, 16, 16), (1000, 64, 8192), (90, 2500, 16400), (2050, 1030, 112), (200, 4090, 4112), (128, 4101, 8208), (333, 5003, 2080),
         (340, 500, 16400), (150, 1001, 16384)]


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_matmul(m, n, k, name):
    torch = torch_dev()
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    x, xs, w, ws = operands(torch, rng, m, n, k)
    xs *= (1024 / k) ** 0.5
    bias = half(torch, rng.normal(0, 1, n), name)[0] if n % 2 else None
    got = []
    for room in (None, torch.full((W.w8_matmul_workspace_bytes(m, n, k) + 16,), 255, dtype=torch.uint8, device="cuda")):
        y = torch.full((m, n), float("nan"), dtype=dtype(torch, name), device="cuda")
        W.w8_matmul(x, xs, w, ws, y, bias=bias, workspace=room)
        check(y, x, xs, w, ws, bias, name)
        got.append(y)
    assert torch.equal(*got), "another workspace gives another result"


@pytest.mark.parametrize("m,n,k", [(3000, 4500, 272), (1024, 16384, 80), (4096, 4096, 1024), (5003, 3001, 160)])
def test_large_tiles(m, n, k):
    torch = torch_dev()
    rng = np.random.default_rng(m + n + k)
    x, xs, w, ws = operands(torch, rng, m, n, k)
    y = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    W.w8_matmul(x, xs, w, ws, y)
    check(y, x, xs, w, ws, None, "bf16")


@pytest.mark.parametrize("m,n,k,tail", [(2048, 2050, 8192, True), (4050, 4352, 8192, True), (4000, 4300, 6160, True),
                                        (7000, 6000, 2064, False), (5000, 9000, 1040, False), (7003, 6003, 1040, False)])
def test_more_tiles_than_compute_units(m, n, k, tail):
    """Workgroups that go on from tile to tile, and last tiles in parts of k: with rows of results at multiples of 16 bytes
    and without, in a workspace, without one, and in one that is a byte too small."""
    torch = torch_dev()
    rng = np.random.default_rng(m * n + k)
    x, xs, w, ws = operands(torch, rng, m, n, k)
    xs *= (1024 / k) ** 0.5
    bias = half(torch, rng.normal(0, 1, n), "fp16")[0]
    need = W.w8_matmul_workspace_bytes(m, n, k)
    assert bool(need) == tail
    room = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    wide = torch.full((m + 2, n + 16), 7.0, dtype=torch.float16, device="cuda")
    first = None
    for space in (room[:need], None, room[:max(need - 1, 0)]):
        wide.fill_(7.0)
        y = wide[1:m + 1, 8:n + 8]
        y.fill_(float("nan"))
        W.w8_matmul(x, xs, w, ws, y, bias=bias, workspace=space)
        if first is None:
            check(y, x, xs, w, ws, bias, "fp16")
            first = y.clone()
        assert torch.equal(first, y), "another workspace gives another result"
        assert (wide[0] == 7).all() and (wide[m + 1] == 7).all() and (wide[:, :8] == 7).all() and (wide[:, n + 8:] == 7).all()
        assert (room[need:] == 255).all()


@pytest.mark.parametrize("m", [1, 20, 64, 65, 200])
def test_against_the_oracle(m):
    torch = torch_dev()
    rng = np.random.default_rng(m)
    x, xs, w, ws = operands(torch, rng, m, 75, 400, low=-128)
    y = torch.empty((m, 75), dtype=torch.float16, device="cuda")
    W.w8_matmul(x, xs, w, ws, y)
    ref = decoder8.product(*(t.cpu().numpy() for t in (x, xs, w, ws)))
    err = 2.0 ** -24 * 3.01 * np.abs(ref)
    assert (np.abs(host(y) - ref) <= err + ROUND["fp16"] * (np.abs(ref) + err) + TINY["fp16"]).all()


@pytest.mark.parametrize("m", [2, 64, 300])
def test_sums_reach_the_end_of_int32(m):
    """The largest k with codes that are all -128, and all of one sign."""
    torch = torch_dev()
    k, n = 131056, 33
    x = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    xs, ws = torch.full((m,), 2.0 ** -16, device="cuda"), torch.full((n,), 2.0 ** -8, device="cuda")
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    W.w8_matmul(x, xs, w, ws, y, workspace=torch.empty(W.w8_matmul_workspace_bytes(m, n, k) + 16, dtype=torch.uint8, device="cuda"))
    check(y, x, xs, w, ws, None, "bf16")


@pytest.mark.parametrize("m", [3, 40, 77, 400])
def test_strided_rows_and_neighbours(m):
    torch = torch_dev()
    rng = np.random.default_rng(m)
    n, k = 70, 208
    x, xs, w, ws = operands(torch, rng, m, n, k + 48)
    wide = torch.full((m + 2, n + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    for left in (0, 1, 8):
        wide.fill_(7.0)
        y = wide[1:m + 1, left:left + n]
        w2 = w[:, :k].contiguous()
        W.w8_matmul(x[:, 16:16 + k], xs, w2, ws, y)
        check(y, x[:, 16:16 + k], xs, w2, ws, None, "bf16")
        assert (wide[0] == 7).all() and (wide[m + 1] == 7).all() and (wide[:, :left] == 7).all() and (wide[:, left + n:] == 7).all()


@pytest.mark.parametrize("m", [4, 64, 150])
def test_rows_that_are_not_numbers(m):
    """A NaN for a scale makes its row, or column, NaN and no other."""
    torch = torch_dev()
    rng = np.random.default_rng(m)
    x, xs, w, ws = operands(torch, rng, m, 50, 96)
    xs[1], ws[7] = float("nan"), float("nan")
    y = torch.zeros((m, 50), dtype=torch.float16, device="cuda")
    W.w8_matmul(x, xs, w, ws, y)
    want = torch.zeros((m, 50), dtype=torch.bool, device="cuda")
    want[1], want[:, 7] = True, True
    assert torch.equal(torch.isnan(y), want)


def test_empty_and_refused():
    torch = torch_dev()
    rng = np.random.default_rng(1)
    x, xs, w, ws = operands(torch, rng, 4, 8, 64)
    y = torch.zeros((4, 8), dtype=torch.bfloat16, device="cuda")
    W.w8_matmul(x[:0], xs[:0], w, ws, y[:0])
    W.w8_matmul(x, xs, w[:0], ws[:0], y[:, :0])
    for rows in (4, 100):
        out = torch.full((rows, 8), 9.0, dtype=torch.bfloat16, device="cuda")
        W.w8_matmul(torch.empty((rows, 0), dtype=torch.int8, device="cuda"), torch.ones(rows, device="cuda"), w[:, :0].contiguous(),
                    ws, out, bias=y[0] + 2)
        assert (out == 2).all()
    for bad in ((x.half(), xs, w, ws, y), (x, xs[:3], w, ws, y), (x, xs, w[:, :32], ws, y), (x, xs, w, ws[:7], y),
                (x, xs, w, ws, y.float()), (x, xs, w, ws, y[:3]), (x, xs.half(), w, ws, y), (x, xs, w.t(), ws, y),
                (x, xs, w, ws, None)):
        with pytest.raises(ValueError):
            W.w8_matmul(*bad)
    with pytest.raises(ValueError):
        W.w8_matmul(x, xs, w, ws, y, bias=y[0].half())
    with pytest.raises(W.WinoError):
        W.w8_matmul(x[:, :40], xs, w[:, :40].contiguous(), ws, y)


def test_rows_past_32_bits():
    """Rows of x and of y that lie further than 2^32 bytes from the first."""
    torch = torch_dev()
    rng = np.random.default_rng(2)
    m, n, k, apart = 70, 48, 64, 1 << 26
    x, xs, w, ws = operands(torch, rng, m, n, k)
    far = torch.empty((m, apart), dtype=torch.int8, device="cuda")
    far[:, :k] = x
    out = torch.empty((m, apart // 2), dtype=torch.float16, device="cuda")
    for rows in (m, 64):
        W.w8_matmul(far[:rows, :k], xs[:rows], w, ws, out[:rows, :n])
        check(out[:rows, :n], x[:rows], xs[:rows], w, ws, None, "fp16")


def test_two_streams_and_graphs():
    """Two graphs that share a workspace, replayed in turn, and calls on two streams with a workspace each."""
    torch = torch_dev()
    rng = np.random.default_rng(4)
    cases = []
    need = 16
    for m, n, k in ((1, 1000, 4096), (24, 512, 8192), (300, 700, 2048)):
        x, xs, w, ws = operands(torch, rng, m, n, k)
        y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        need = max(need, W.w8_matmul_workspace_bytes(m, n, k) + 16)
        cases.append((x, xs, w, ws, y))
    room = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = []
    for x, xs, w, ws, y in cases:
        W.w8_matmul(x, xs, w, ws, y, workspace=room[0])
        want.append(y.clone())
    graphs = []
    side = torch.cuda.Stream()
    for x, xs, w, ws, y in cases:
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            W.w8_matmul(x, xs, w, ws, y, workspace=room[0])
        graphs.append(g)
    for _ in range(3):
        for g, c, ref in zip(graphs, cases, want):
            c[4].zero_()
            g.replay()
            assert torch.equal(c[4], ref)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cases:
        c[4].zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        for i, (x, xs, w, ws, y) in enumerate(cases):
            W.w8_matmul(x, xs, w, ws, y, workspace=room[i % 2], stream=streams[i % 2])
    torch.cuda.synchronize()
    for c, ref in zip(cases, want):
        assert torch.equal(c[4], ref)

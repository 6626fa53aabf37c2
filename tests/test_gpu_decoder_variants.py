"""The decoder operators at the sizes where another kernel, tile or split of
the work takes over; the bounds are those of each operator's own tests."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder

from decoder_util import ROUND, attention_bound, dtype, half, host
from gpu_util import torch_dev
from test_gpu_kv4_append import _run as append_run
from test_gpu_kv4_attention import _call, _hold, _setup, _workspace
from test_gpu_kv4_attention import _reference as decode_reference
from test_gpu_prompt_attention import _cu
from test_gpu_prompt_attention import _reference as prompt_reference
from test_gpu_w4_matvec import _check

pytestmark = pytest.mark.gpu


def _check_rounded(y, x, w, b, name):
    """_check, which speaks of results on either side of the largest number of
    fp16, and of those that may lie between: a sum, off by `err` at most, that
    reaches 65520, halfway to 2^16, rounds to infinity."""
    if name == "fp16":
        ref = x @ w.T + (0 if b is None else b)
        err = (x.shape[1] + 1) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b)))
        between = (np.abs(ref) + err >= 65520) & (np.abs(ref) - err <= 65536 * (1 + ROUND[name]))
        assert (between & (y == np.sign(ref) * np.inf) | (np.abs(y - ref) <= err + 32) | ~between).all()
        keep = ~between
        for i in range(len(y)):
            _check(y[i:i + 1, keep[i]], x[i:i + 1], w[keep[i]], None if b is None else b[keep[i]], name)
    else:
        _check(y, x, w, b, name)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("lowest,highest", [(104, 140), (98, 146)])
@pytest.mark.parametrize("m,n,k", [
    (3, 80, 1056),                                     # x in LDS: few rows of W,
    (2, 5000, 96), (1, 8300, 160),                     # more, many
    (16, 200, 1312), (16, 4200, 1312), (16, 8210, 1312),  # x beside the codes, the same
    (3, 100, 8192), (9, 2100, 8224), (1, 70, 12320),   # a long k in parts
    (20, 40, 1056), (20, 2100, 2080), (32, 4100, 96),  # two tiles of x
    (35, 40, 4128), (33, 2060, 2112), (66, 2100, 32)])  # four
def test_matvec_cuts(m, n, k, lowest, highest, name):
    """Scales of a row within a factor of 16, rows over the whole range: with x in
    fp16, rows of tiny weights, of large ones, and of ones that fp16 does not hold."""
    torch = torch_dev()
    rng = np.random.default_rng(m + 3 * n + 7 * k + highest)
    codes = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
    base = rng.integers(lowest, highest - 3, (n, 1))
    base[:2, 0] = lowest, highest - 4
    scales = (base + rng.integers(0, 5, (n, k // 32))).astype(np.uint8)
    w = decoder.decode(codes, scales)
    x, xv = half(torch, rng.normal(0, 1, (m, k)), name)
    bias, bv = half(torch, rng.normal(0, 1, n), name) if k % 64 else (None, None)
    cd, sd = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    for ws in (torch.full((W.w4_matvec_workspace_bytes(m, n, k) + 16,), 255, dtype=torch.uint8, device="cuda"), None):
        got = []
        for _ in range(2):
            y = torch.full((m, n), float("nan"), dtype=dtype(torch, name), device="cuda")
            W.w4_matvec(x, cd, sd, y, bias=bias, workspace=ws)
            got.append(host(y))
        _check_rounded(got[0], xv, w, bv, name)
        assert (got[0] == got[1]).all(), "the same call gives another result"


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", [(12, 1000, 8224), (6, 8300, 1312), (5, 8200, 160), (20, 40, 1312), (18, 300, 4640),
                                   (18, 9000, 160), (17, 8200, 2624), (40, 4200, 128), (35, 300, 5152), (50, 8250, 544),
                                   (70, 33, 1600), (64, 4100, 1024)])
def test_matmul_far_apart_rows_and_not_finite(m, n, k, name):
    """Rows of x within a wider tensor, the last columns of two of them not
    finite: their own outputs are not numbers or infinite, the others' ordinary,
    whatever is read past the ends of k and m."""
    torch = torch_dev()
    rng = np.random.default_rng(m + n + k)
    codes = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
    scales = rng.integers(120, 130, (n, k // 32), dtype=np.uint8)
    w = decoder.decode(codes, scales)
    wide, wv = half(torch, rng.normal(0, 1, (m, k + 24)), name)
    x, xv = wide[:, 8:8 + k], wv[:, 8:8 + k]
    x[3, k - 1], x[m - 1, k - 1] = float("nan"), float("inf")
    wide[:, :8] = wide[:, 8 + k:] = float("nan")
    cd, sd = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    zero = (codes[:, -1] >> 4 & 7) == 0
    keep = [i for i in range(m) if i not in (3, m - 1)]
    for ws in (torch.full((W.w4_matvec_workspace_bytes(m, n, k) + 16,), 255, dtype=torch.uint8, device="cuda"), None):
        y = torch.full((m, n), 3.0, dtype=dtype(torch, name), device="cuda")
        W.w4_matvec(x, cd, sd, y, workspace=ws)
        got = host(y)
        assert np.isnan(got[3]).all() and np.isnan(got[m - 1][zero]).all() and np.isinf(got[m - 1][~zero]).all()
        _check_rounded(got[keep], xv[keep], w, None, name)


@pytest.mark.parametrize("m,n,k", [(3, 70, 96), (20, 300, 1312)])
def test_matvec_infinity_times_weights_past_fp16(m, n, k):
    """An infinite x with weights that fp16 does not hold: infinite, not NaN."""
    torch = torch_dev()
    rng = np.random.default_rng(71)
    codes = rng.integers(0, 256, (n, k // 2), dtype=np.uint8) | 0x22          # no weight is zero
    scales = np.full((n, k // 32), 98, np.uint8)
    x, xv = half(torch, rng.normal(0, 1, (m, k)), "fp16")
    x[1, 40] = float("-inf")
    y = torch.zeros((m, n), dtype=torch.float16, device="cuda")
    W.w4_matvec(x, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), y)
    got, w = host(y), decoder.decode(codes, scales)
    assert (got[1] == -np.sign(w[:, 40]) * np.inf).all()
    _check(np.delete(got, 1, 0), np.delete(xv, 1, 0), w, None, "fp16")


def test_matvec_cuts_into_parts():
    """The sizes above do reach the parts."""
    assert W.w4_matvec_workspace_bytes(3, 100, 8192) > 0 and W.w4_matvec_workspace_bytes(9, 2100, 8224) > 0
    assert W.w4_matvec_workspace_bytes(1, 70, 12320) > 0 and W.w4_matvec_workspace_bytes(33, 2060, 2112) > 0


@pytest.mark.parametrize("name,pairs", [("bf16", False), ("fp16", True)])
def test_append_large_outputs(name, pairs):
    torch = torch_dev()
    append_run(torch, np.random.default_rng(51), 1030, 256, 1, 64, 64, pairs, 16, name, W.KV4_CACHED)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d,q_len,hq,hkv", [(64, 1, 8, 2), (96, 3, 12, 1), (128, 2, 20, 2), (192, 1, 5, 1), (256, 5, 4, 1)])
def test_decode_many_sequences_over_a_long_table(d, q_len, hq, hkv, name):
    """Shares of several sequences, sequences of several shares, ones with nothing,
    and groups of heads that need more than one tile."""
    torch = torch_dev()
    rng = np.random.default_rng(d + q_len)
    lens = [int(x) for x in rng.integers(0, 90, 70)]
    lens[0], lens[7], lens[8], lens[31], lens[69] = 0, 2900, 256, 1025, 1300
    page = 32
    table, cache, q, qv = _setup(torch, rng, lens, q_len, hq, hkv, d, page, name)
    ws = _workspace(torch, lens, q_len, hq, hkv, d, table, page)
    assert ws.numel() > 16
    got = host(_call(torch, q, cache, table, lens, d ** -0.5, ws))
    ref, bound = decode_reference(cache, table, lens, qv, q_len, hq, hkv, d, page, d ** -0.5, name)
    _hold(got, ref, bound)
    assert (host(_call(torch, q, cache, table, lens, d ** -0.5, ws)) == got).all(), "not the same twice"


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hkv", [(64, 32, 16), (96, 16, 16), (128, 16, 16), (192, 16, 8), (256, 16, 16)])
def test_prompt_many_sequences(d, hq, hkv, causal, name):
    """Enough sequences to fill the device, of ragged lengths, some without
    queries or keys, with more and with fewer keys than queries."""
    torch = torch_dev()
    rng = np.random.default_rng(d + hq)
    seqs = 44
    q_lens = [int(x) for x in rng.integers(1, 9, seqs)]
    k_lens = [n + int(x) for n, x in zip(q_lens, rng.integers(0, 70, seqs))]
    q_lens[3], k_lens[3], q_lens[5], k_lens[9], q_lens[20], k_lens[20] = 0, 5, 9, 0, 70, 33
    q_lens[43], k_lens[43] = 131, 260
    q, qv = half(torch, rng.normal(0, 1, (sum(q_lens), hq, d)), name)
    k, kv = half(torch, rng.normal(0, 1.5, (sum(k_lens), hkv, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (sum(k_lens), hkv, d)), name)
    ref, bound = prompt_reference(qv, kv, vv, q_lens, k_lens, d ** -0.5, causal, name)
    cu_q, cu_k = _cu(torch, q_lens), _cu(torch, k_lens)
    got = []
    for hint in (131, 1, 131):
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, cu_q, cu_k, hint, out, d ** -0.5, causal=causal)
        got.append(host(out))
        _hold(got[-1], ref, bound)
    assert (got[0] == got[2]).all(), "not the same twice"


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prompt_many_sequences_one_value_not_finite(d, bad):
    """A value that is not finite reaches the queries that see its token, in its own dimension, and nothing else."""
    torch = torch_dev()
    rng = np.random.default_rng(d)
    lens, heads = [9] * 40 + [70], 16
    q, qv = half(torch, rng.normal(0, 1, (sum(lens), heads, d)), "bf16")
    k, kv = half(torch, rng.normal(0, 1, (sum(lens), heads, d)), "bf16")
    v, vv = half(torch, rng.normal(0, 1, (sum(lens), heads, d)), "bf16")
    ref, bound = prompt_reference(qv, kv, vv, lens, lens, 0.1, True, "bf16")
    hit = np.zeros(q.shape, bool)
    for at, end in ((4, 9), (360 + 50, 430)):
        v[at, 5, 33] = bad
        hit[at:end, 5, 33] = True
    out = torch.zeros_like(q)
    W.prompt_attention(q, k, v, _cu(torch, lens), _cu(torch, lens), 70, out, 0.1)
    got = host(out)
    _hold(got[~hit], ref[~hit], bound[~hit])
    assert (np.isnan(got[hit]) if np.isnan(bad) else got[hit] == bad).all()


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_prompt_few_queries_on_many_keys(d, name):
    torch = torch_dev()
    rng = np.random.default_rng(d + 1)
    q_lens, k_lens, hq, hkv = [37, 1], [2105, 131], 6, 2
    q, qv = half(torch, 2 * rng.normal(0, 1, (sum(q_lens), hq, d)), name)
    k, kv = half(torch, rng.normal(0, 1, (sum(k_lens), hkv, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (sum(k_lens), hkv, d)), name)
    for causal in (True, False):
        ref, bound = prompt_reference(qv, kv, vv, q_lens, k_lens, d ** -0.5, causal, name)
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, _cu(torch, q_lens), _cu(torch, k_lens), 37, out, d ** -0.5, causal=causal)
        _hold(host(out), ref, bound)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [128, 192, 256])
def test_prompt_maxima_that_keep_growing(d, name):
    """Keys that grow along the sequence, so that the largest score is outgrown
    again and again, in one wave or another; a sample of the rows."""
    torch = torch_dev()
    rng = np.random.default_rng(d + 5)
    lens, heads = [700, 690, 701, 650], 16
    n = sum(lens)
    grow = np.concatenate([np.linspace(0.1, 4, m) for m in lens])[:, None, None]
    q, qv = half(torch, 3 * rng.normal(0, 1, (n, heads, d)), name)
    k, kv = half(torch, grow * rng.normal(0, 1, (n, heads, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (n, heads, d)), name)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    W.prompt_attention(q, k, v, _cu(torch, lens), _cu(torch, lens), max(lens), out, d ** -0.5)
    got = host(out)
    begin = 0
    for m in lens:
        for i in [0, 31, 32, 63, 64, 127, 128, m - 1] + list(range(50, m, 113)):
            for h in (0, 7, 15):
                r, w, z = decoder.attend(qv[begin + i, h], kv[begin:begin + m, h], vv[begin:begin + m, h],
                                         np.arange(i + 1), d ** -0.5)
                _hold(got[begin + i, h], r, attention_bound(r, w, z, i + 1, d, name, ROUND[name]))
        begin += m


def test_prompt_offsets_that_fall():
    """Offsets below 0 and falling ones, down to the type's lowest value: such
    sequences are empty, the others are not touched by it."""
    torch = torch_dev()
    rng = np.random.default_rng(62)
    n, hq, hkv, d = 60, 4, 2, 64
    q, qv = half(torch, rng.normal(0, 1, (n, hq, d)), "bf16")
    k, kv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    v, vv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    low = -2 ** 31
    cu_q = torch.tensor([5, 25, low, -1, 0], dtype=torch.int32, device="cuda")
    cu_k = torch.tensor([7, 47, low, 3, -9], dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    W.prompt_attention(q, k, v, cu_q, cu_k, 20, out, 0.1)
    ref, bound = prompt_reference(qv[5:25], kv[7:47], vv[7:47], [20], [40], 0.1, True, "bf16")
    _hold(host(out)[5:25], ref, bound)
    assert (out[:5] == 7).all() and (out[25:] == 7).all()


def test_prompt_rows_far_apart():
    """Keys and values whose offsets pass 32 bits, in elements as well."""
    torch = torch_dev()
    rng = np.random.default_rng(61)
    n, hq, hkv, d, stride = 300, 2, 1, 128, 1 << 24
    big = torch.empty(((n - 1) * stride + 4096,), dtype=torch.bfloat16, device="cuda")
    assert big.numel() > 1 << 32
    k, v = (big[o:].as_strided((n, hkv, d), (stride, d, 1)) for o in (0, 2048))
    q, qv = half(torch, rng.normal(0, 1, (n, hq, d)), "bf16")
    kt, kv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    vt, vv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    k.copy_(kt)
    v.copy_(vt)
    out = torch.zeros_like(q)
    W.prompt_attention(q, k, v, _cu(torch, [n]), _cu(torch, [n]), n, out, 0.1)
    ref, bound = prompt_reference(qv, kv, vv, [n], [n], 0.1, True, "bf16")
    _hold(host(out), ref, bound)


def test_what_is_no_tensor_is_refused():
    torch = torch_dev()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    u8, i32 = torch.uint8, torch.int32
    x, c, s, y = z(2, 64), z(8, 32, dt=u8), z(8, 2, dt=u8), z(2, 8)
    q, k, cu = z(4, 2, 64), z(4, 1, 64), z(2, dt=i32)
    cache = (z(2, 1, 16, 32, dt=u8), z(2, 1, 16, 2, dt=u8)) * 2
    for bad in (None, 3, "x", np.zeros((2, 64), np.float16), [1.0]):
        for call in (lambda: W.w4_matvec(bad, c, s, y), lambda: W.w4_matvec(x, bad, s, y),
                     lambda: W.w4_matvec(x, c, s, bad),
                     lambda: W.prompt_attention(bad, k, k, cu, cu, 4, q, 1.0),
                     lambda: W.prompt_attention(q, k, k, bad, cu, 4, q, 1.0),
                     lambda: W.kv4_attention(bad, cache, z(1, 2, dt=i32), z(1, dt=i32), z(1, 2, 64), 1.0),
                     lambda: W.kv4_attention(z(1, 2, 64), bad, z(1, 2, dt=i32), z(1, dt=i32), z(1, 2, 64), 1.0),
                     lambda: W.kv4_append(None, bad, k, z(8, 64, dt=torch.float32), z(4, dt=i32),
                                          z(4, dt=torch.int64), cache)):
            with pytest.raises((ValueError, TypeError)):
                call()


@pytest.mark.parametrize("d,hq,hkv,seqs", [(64, 2, 1, 65), (128, 16, 8, 130), (256, 4, 4, 200), (64, 1, 1, 1000)])
def test_prompt_more_sequences_than_a_wave(d, hq, hkv, seqs):
    """Sequences are ranked 64 at a time: several such groups, with empty sequences and ones without keys in each."""
    torch = torch_dev()
    rng = np.random.default_rng(seqs)
    q_lens = [int(x) for x in rng.integers(0, 5, seqs)]
    k_lens = [max(0, n + int(x)) for n, x in zip(q_lens, rng.integers(-3, 20, seqs))]
    q_lens[63], k_lens[63], q_lens[64], k_lens[64], q_lens[-1], k_lens[-1] = 140, 150, 0, 9, 3, 80
    q, qv = half(torch, rng.normal(0, 1, (sum(q_lens), hq, d)), "bf16")
    k, kv = half(torch, rng.normal(0, 1.5, (sum(k_lens), hkv, d)), "bf16")
    v, vv = half(torch, rng.normal(0, 1, (sum(k_lens), hkv, d)), "bf16")
    ref, bound = prompt_reference(qv, kv, vv, q_lens, k_lens, d ** -0.5, True, "bf16")
    for hint in (140, 100000):
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, _cu(torch, q_lens), _cu(torch, k_lens), hint, out, d ** -0.5)
        _hold(host(out), ref, bound)


@pytest.mark.parametrize("seqs,hq,hkv,offset", [(5000, 1, 1, 0), (130, 6, 2, 40), (64, 6, 2, 40), (8300, 2, 1, 3)])
def test_prompt_sets_of_sequences_are_found(seqs, hq, hkv, offset):
    """Thousands of sequences, of no tokens to 300, rows before the first one and offsets past the last row."""
    torch = torch_dev()
    rng = np.random.default_rng(seqs)
    d = 64
    lens = rng.integers(0, 3, seqs)
    lens[[0, seqs // 2, seqs - 1]] = 3, 300, 70
    cu = (offset + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)
    n = int(cu[-1]) - (20 if offset else 0)                       # the last sequence is cut off
    cut = np.minimum(cu, n)
    q, qv = half(torch, rng.normal(0, 1, (n, hq, d)), "bf16")
    k, kv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    v, vv = half(torch, rng.normal(0, 1, (n, hkv, d)), "bf16")
    got_lens = [int(x) for x in np.diff(cut)]
    ref, bound = prompt_reference(qv[offset:], kv[offset:], vv[offset:], got_lens, got_lens, 0.1, True, "bf16")
    t = torch.from_numpy(cu).cuda()
    for hint in (300, 3, 1 << 20):
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, t, t, hint, out, 0.1)
        _hold(host(out)[offset:], ref, bound)
        assert (out[:offset] == 7).all()


def test_prompt_work_grows_with_the_sequences_not_their_square():
    """Sixteen times as many sequences take about sixteen times as long; looking at all of them in each workgroup took
    a hundred and thirty times as long."""
    torch = torch_dev()

    def time(seqs):
        q = torch.zeros((4 * seqs, 16, 128), dtype=torch.bfloat16, device="cuda")
        k, out = q[:, :4], torch.empty_like(q)
        cu = (4 * torch.arange(seqs + 1, device="cuda")).to(torch.int32)
        took = []
        for _ in range(6):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            for _ in range(4):
                W.prompt_attention(q, k, k, cu, cu, 4, out, 0.1)
            end.record()
            torch.cuda.synchronize()
            took.append(begin.elapsed_time(end))
        return min(took)

    few, many = time(256), time(4096)
    assert many < 50 * few, (few, many)

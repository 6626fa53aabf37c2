"""prompt_attention against softmax attention in float64, sequence by
sequence.  Element-wise bound: decoder_util.attention_bound, with
probabilities rounded to the 16-bit type for the matrix cores."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder

from decoder_util import ROUND, attention_bound, dtype, half, host
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def _reference(qv, kv, vv, q_lens, k_lens, scale, causal, name):
    hq, d = qv.shape[1:]
    hkv = kv.shape[1]
    ref, bound = np.zeros(qv.shape), np.zeros(qv.shape)
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        for h in range(hq):
            k, v = (x[k0:k0 + nk, h * hkv // hq] for x in (kv, vv))
            for i in range(nq):
                seen = np.arange(max(0, nk - nq + 1 + i) if causal else nk)
                r, w, s = decoder.attend(qv[q0 + i, h], k, v, seen, scale)
                ref[q0 + i, h] = r
                bound[q0 + i, h] = attention_bound(r, w, s, len(seen), d, name, ROUND[name])
        q0, k0 = q0 + nq, k0 + nk
    return ref, bound


def _cu(torch, lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def _hold(got, ref, bound):
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {ref[bad][0]} +- {bound[bad][0]}")


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lens,k_lens,hq,hkv,d", [
    ([1], [1], 1, 1, 64), ([2, 0, 5], [2, 0, 5], 4, 2, 64), ([33, 31, 64, 1], None, 2, 1, 128),
    ([129], None, 3, 3, 128), ([65, 127, 3], None, 4, 1, 96), ([100], [163], 2, 2, 192), ([40, 70], [10, 70], 2, 1, 256),
    ([5, 7, 9], [0, 200, 9], 6, 2, 128), ([260], None, 2, 1, 64), ([1, 1, 1], [300, 2, 64], 8, 2, 128),
    ([66, 130], [200, 131], 5, 1, 96)])
def test_prompt(q_lens, k_lens, hq, hkv, d, causal, name):
    torch = torch_dev()
    k_lens = q_lens if k_lens is None else k_lens
    rng = np.random.default_rng(sum(q_lens) + 7 * sum(k_lens) + d + hq)
    q, qv = half(torch, rng.normal(0, 1, (sum(q_lens), hq, d)), name)
    k, kv = half(torch, rng.normal(0, 1.5, (sum(k_lens), hkv, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (sum(k_lens), hkv, d)), name)
    ref, bound = _reference(qv, kv, vv, q_lens, k_lens, d ** -0.5, causal, name)
    cu_q, cu_k = _cu(torch, q_lens), _cu(torch, k_lens)
    got = []
    for hint in (max(q_lens), 1, 100000):                     # a hint: any value gives a right result
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, cu_q, cu_k, hint, out, d ** -0.5, causal=causal)
        got.append(host(out))
        _hold(got[-1], ref, bound)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    W.prompt_attention(q, k, v, cu_q, cu_k, 100000, out, d ** -0.5, causal=causal)
    assert (host(out) == got[-1]).all(), "not the same twice"


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_longer(d, name):
    """Several tiles in each direction and peaked scores, a sample of the rows."""
    torch = torch_dev()
    rng = np.random.default_rng(d)
    n, hq, hkv = 1111, 2, 1
    q, qv = half(torch, 3 * rng.normal(0, 1, (n, hq, d)), name)
    k, kv = half(torch, rng.normal(0, 1, (n, hkv, d)), name)
    v, vv = half(torch, rng.normal(0, 1, (n, hkv, d)), name)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    cu = _cu(torch, [n])
    W.prompt_attention(q, k, v, cu, cu, n, out, d ** -0.5)
    got = host(out)
    for i in list(range(0, n, 37)) + [63, 64, 127, 128, 255, 256, 1023, 1024, n - 1]:
        for h in range(hq):
            r, w, s = decoder.attend(qv[i, h], kv[:, 0], vv[:, 0], np.arange(i + 1), d ** -0.5)
            _hold(got[i, h], r, attention_bound(r, w, s, i + 1, d, name, ROUND[name]))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("which", ["k", "v"])
def test_prompt_not_finite_reaches_only_who_sees_it(which, bad):
    """A key or value that is not finite: earlier queries of its sequence, and
    other sequences in the same tile, get their ordinary results."""
    torch = torch_dev()
    rng = np.random.default_rng(31)
    lens, hq, hkv, d = [20, 75, 30], 2, 1, 128
    q, qv = half(torch, rng.normal(0, 1, (sum(lens), hq, d)), "bf16")
    k, kv = half(torch, rng.normal(0, 1, (sum(lens), hkv, d)), "bf16")
    v, vv = half(torch, rng.normal(0, 1, (sum(lens), hkv, d)), "bf16")
    ref, bound = _reference(qv, kv, vv, lens, lens, 0.09, True, "bf16")
    at = 20 + 41
    (k if which == "k" else v)[at, 0, 77] = bad
    out = torch.zeros_like(q)
    W.prompt_attention(q, k, v, _cu(torch, lens), _cu(torch, lens), 75, out, 0.09)
    got = host(out)
    hit = np.zeros(got.shape, bool)
    hit[at:95, :, 77] = True
    if which == "k":
        hit[at:95] = True
        if bad == float("inf") or bad == float("-inf"):
            hit[at:95] = True                                   # +-inf scores: NaN, or a key that counts for nothing
            fine = np.isnan(got[at:95]).all(-1) | np.isfinite(got[at:95]).all(-1)
            assert fine.all()
            up = np.sign(qv[at:95, :, 77]) == np.sign(bad)
            assert np.isnan(got[at:95][up]).all()
        else:
            assert np.isnan(got[hit]).all()
    elif np.isnan(bad):
        assert np.isnan(got[hit]).all()
    else:
        assert (got[hit] == bad).all()
    _hold(got[~hit], ref[~hit], bound[~hit])


def test_prompt_slices_rows_without_a_sequence_and_offsets_past_the_end():
    """q, k, v as slices of one projection's output; rows that no sequence covers
    stay as they were; offsets past the tensors are cut off."""
    torch = torch_dev()
    rng = np.random.default_rng(32)
    n, hq, hkv, d = 90, 4, 2, 64
    x, xv = half(torch, rng.normal(0, 1, (n, hq + 2 * hkv, d)), "bf16")
    q, k, v = x.split((hq, hkv, hkv), 1)
    qv, kv, vv = xv[:, :hq], xv[:, hq:hq + hkv], xv[:, hq + hkv:]
    out = torch.full((n, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([10, 40, 80], dtype=torch.int32, device="cuda")
    W.prompt_attention(q, k, v, cu, cu, 40, out, 0.125)
    ref, bound = _reference(qv[10:80], kv[10:80], vv[10:80], [30, 40], [30, 40], 0.125, True, "bf16")
    _hold(host(out)[10:80], ref, bound)
    assert (out[:10] == 7).all() and (out[80:] == 7).all()
    far = torch.tensor([10, 40, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ref, bound = _reference(qv[10:], kv[10:], vv[10:], [30, 50], [30, 50], 0.125, False, "bf16")
    W.prompt_attention(q, k, v, far, far, 40, out, 0.125, causal=False)
    _hold(host(out)[10:], ref, bound)


def test_prompt_scales_and_empty_calls():
    torch = torch_dev()
    rng = np.random.default_rng(33)
    n, hq, hkv, d = 70, 2, 1, 128
    q, qv = half(torch, rng.normal(0, 1, (n, hq, d)), "fp16")
    k, kv = half(torch, rng.normal(0, 1, (n, hkv, d)), "fp16")
    v, vv = half(torch, rng.normal(0, 1, (n, hkv, d)), "fp16")
    cu = _cu(torch, [n])
    for scale in (0.0, -0.2, 5.0):
        ref, bound = _reference(qv, kv, vv, [n], [n], scale, True, "fp16")
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        W.prompt_attention(q, k, v, cu, cu, n, out, scale)
        _hold(host(out), ref, bound)
    none = cu[:1] * 0
    out = torch.full_like(q, 4.0)
    W.prompt_attention(q, k, v, none, none, 0, out, 1.0)                            # no sequences
    W.prompt_attention(q[:0], k, v, cu * 0, cu * 0, 0, out[:0], 1.0)                # no rows
    assert (out == 4).all()
    W.prompt_attention(q, k[:0], v[:0], cu, cu * 0, n, out, 1.0)                    # no keys at all
    assert (out == 0).all()


def test_prompt_in_a_graph_and_on_another_stream():
    torch = torch_dev()
    rng = np.random.default_rng(34)
    lens, hq, hkv, d = [150, 3, 260], 4, 2, 128
    n = sum(lens)
    q, k, v = (half(torch, rng.normal(0, 1, (n, h, d)), "bf16")[0] for h in (hq, hkv, hkv))
    cu, out = _cu(torch, lens), torch.zeros_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    W.prompt_attention(q, k, v, cu, cu, 260, out, 0.1, stream=side)
    side.synchronize()
    eager = torch.zeros_like(q)
    W.prompt_attention(q, k, v, cu, cu, 260, eager, 0.1)
    assert torch.equal(out, eager) and float(out.abs().sum()) > 0
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        W.prompt_attention(q, k, v, cu, cu, 260, out, 0.1)
    for i in range(3):
        q.copy_(half(torch, rng.normal(0, 1 + i, (n, hq, d)), "bf16")[0])
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        W.prompt_attention(q, k, v, cu, cu, 260, eager, 0.1)
        assert torch.equal(out, eager)


def test_prompt_refuses_other_tensors():
    torch = torch_dev()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    q, k, cu = z(8, 4, 64), z(8, 2, 64), torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    W.prompt_attention(q, k, k, cu, cu, 8, z(8, 4, 64), 1.0)
    for bad in (lambda: W.prompt_attention(q.float(), k, k, cu, cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k.half(), k, cu, cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k, k[:4], cu, cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k[..., :32], k, cu, cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k, k, cu.long(), cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k, k, cu, cu[:1], 8, q, 1.0),
                lambda: W.prompt_attention(q, k, k, cu, cu, 8, q[:4], 1.0),
                lambda: W.prompt_attention(q.cpu(), k, k, cu, cu, 8, q, 1.0),
                lambda: W.prompt_attention(q, k.transpose(0, 1).contiguous().transpose(0, 1), k, cu, cu, 8, q, 1.0)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: W.prompt_attention(z(8, 3, 64), k, k, cu, cu, 8, z(8, 3, 64), 1.0), -1),
                        (lambda: W.prompt_attention(q, k, k, cu, cu, 8, z(8, 4, 64), float("inf")), -1),
                        (lambda: W.prompt_attention(z(8, 4, 80), z(8, 2, 80), z(8, 2, 80), cu, cu, 8, z(8, 4, 80), 1.0), -2)):
        with pytest.raises(W.WinoError) as e:
            bad()
        assert e.value.status == status

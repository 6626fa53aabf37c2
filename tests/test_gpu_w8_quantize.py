"""w8_quantize against exact rationals: codes are equal, scales are the exact
ones rounded once to fp32."""
import numpy as np
import pytest

import paper_2209_12982_amd as W
from oracle import decoder8

from decoder_util import dtype, half
from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def _run(torch, x):
    m, k = x.shape
    codes = torch.full((m, k), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((m,), -1.0, device="cuda")
    W.w8_quantize(x, codes, scales)
    return codes.cpu().numpy().astype(np.int64), scales.cpu().numpy()


def _check(xv, codes, scales):
    for i, row in enumerate(xv):
        want, scale = decoder8.quantize_row(row)
        assert (codes[i] == want).all(), i
        # one rounding to fp32, subnormal numbers included; float(Fraction) rounds to 53 bits first, which moves no quotient
        # by 127 across a fp32 rounding point: such a quotient has a period of 7 bits and never 29 equal ones in a row
        assert scales[i] == np.float32(float(scale)), i


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("m,k", [(1, 16), (3, 48), (5, 1024), (2, 2080), (2, 4096), (3, 4112), (1, 16384), (1, 16400), (2, 40000)])
def test_quantize(m, k, name):
    torch = torch_dev()
    rng = np.random.default_rng(m * 31 + k)
    x, xv = half(torch, rng.normal(0, 1, (m, k)) * np.exp(rng.normal(0, 1, k)), name)
    _check(xv, *_run(torch, x))


@pytest.mark.parametrize("name", ["bf16", "fp16"])
def test_halves_and_ends_of_the_range(name):
    """Quotients that lie half-way between codes, rows of the smallest and the largest numbers, zeros."""
    torch = torch_dev()
    rng = np.random.default_rng(3)
    rows = [np.arange(-127, 128) / 2 * 2.0 ** e for e in (0, -7, 5)]
    rows = [np.concatenate([r, [-127 * 2.0 ** e], np.zeros(0)]) for r, e in zip(rows, (0, -7, 5))]     # max 127: code = value
    rows.append(np.linspace(-1, 1, 256))
    small, large = (2.0 ** -133, 3.38e38) if name == "bf16" else (2.0 ** -24, 65504.0)
    rows.append(rng.integers(-9, 10, 256) * small)
    rows.append(np.where(rng.random(256) < 0.02, small, 0))
    rows.append(rng.uniform(-1, 1, 256) * large)
    rows.append(np.zeros(256))
    rows.append(np.where(np.arange(256) == 17, -large, small))
    if name == "bf16":
        rows.append(rng.uniform(-1, 1, 256) * 2.0 ** -64)
        rows.append(rng.uniform(-1, 1, 256) * 2.0 ** -65)
    x, xv = half(torch, np.stack(rows), name)
    _check(xv, *_run(torch, x))


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("k", [32, 5008, 20000])
def test_rows_that_are_not_finite(k, name):
    torch = torch_dev()
    rng = np.random.default_rng(k)
    x, xv = half(torch, rng.normal(0, 1, (5, k)), name)
    x[0, k - 1], x[2, 3], x[4, k // 2] = float("inf"), float("nan"), float("-inf")
    codes, scales = _run(torch, x)
    assert np.isnan(scales[[0, 2, 4]]).all() and (codes[[0, 2, 4]] == 0).all()
    _check(xv[[1, 3]], codes[[1, 3]], scales[[1, 3]])


def test_strided_rows_streams_and_neighbours():
    torch = torch_dev()
    rng = np.random.default_rng(9)
    whole, values = half(torch, rng.normal(0, 1, (7, 320)), "fp16")
    x = whole[:, 64:64 + 176]
    memory = torch.full((7 * 176 + 32,), 55, dtype=torch.int8, device="cuda")
    codes = memory[16:16 + 7 * 176].view(7, 176)
    scales = torch.full((9,), 3.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    W.w8_quantize(x, codes, scales[1:8], stream=side)
    side.synchronize()
    _check(values[:, 64:240], codes.cpu().numpy().astype(np.int64), scales[1:8].cpu().numpy())
    assert (memory[:16] == 55).all() and (memory[16 + 7 * 176:] == 55).all() and scales[0] == 3 and scales[8] == 3


def test_empty_and_refused():
    torch = torch_dev()
    for m, k in ((0, 64), (3, 0)):
        scales = torch.full((m,), 5.0, device="cuda")
        W.w8_quantize(torch.empty((m, k), dtype=torch.bfloat16, device="cuda"), torch.empty((m, k), dtype=torch.int8, device="cuda"),
                      scales)
        assert (scales == 0).all()
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    for bad in ((x.float(), codes, scales), (x, codes.int(), scales), (x, codes, scales[:3]), (x, codes[:3], scales),
                (x.t(), codes, scales), (x, codes, scales.half()), (x, None, scales), (x[:, ::2], codes[:, :32], scales)):
        with pytest.raises(ValueError):
            W.w8_quantize(*bad)
    with pytest.raises(W.WinoError):
        W.w8_quantize(x[:, :40], torch.zeros((4, 40), dtype=torch.int8, device="cuda"), scales)
    assert dtype(torch, "bf16") == x.dtype

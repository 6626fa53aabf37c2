"""Helpers of the 4-bit decoder operators' tests: types, rounding bounds, and
the pieces that build a paged cache (no arithmetic of the operators)."""
import numpy as np

# unit roundoff of the 16-bit types and half their smallest subnormal
ROUND = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}


def dtype(torch, name):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def half(torch, a, name):
    """numpy -> (GPU tensor of the 16-bit type, the float64 values it holds)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dtype(torch, name)).cuda()
    return t, t.double().cpu().numpy()


def host(t):
    return t.double().cpu().numpy()


def attention_bound(ref, weight, score, n, d, name, eps_p):
    """Largest |error| of one output element.  `weight` = sum p|v|, `score` the
    largest scale * sum|q||k|.  A score of d products in fp32 (and its scaling)
    is off by at most delta = (d + 8) 2^-23 score; a probability then by a
    factor 1 +- (2 delta + 2^-21 for the exponential), and eps_p more where it is
    rounded for the matrix cores; the two sums of n terms by n 2^-23 each; the
    result is rounded once."""
    delta = (d + 8) * 2.0 ** -23 * score
    rel = 4 * delta + 2 * eps_p + 2.0 ** -19 + 2 * n * 2.0 ** -23
    err = rel * weight
    return err + ROUND[name] * (np.abs(ref) + err) + TINY[name]


def paged(rng, lens, page, extra=2):
    """A table of distinct pages in random order for sequences of `lens` tokens."""
    counts = [-(-n // page) for n in lens]
    total = sum(counts) + extra
    order = rng.permutation(total)
    table = np.full((len(lens), max(max(counts, default=0), 1)), -1, np.int32)
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total

"""The example decoder: tokens decoded one at a time get the logits that they
get as part of a prompt, and the captured step gives what the eager one gives.

Prompt and steps round alike except in the order of sums and in the
probabilities, so values differ by a few 2^-9 of themselves; a key or value that
lies within that of the middle between two codes (one in fifty or so) may then
go to the other one, a quarter of its size away.  That makes the scores and the
attention's outputs differ by some 0.25 / sqrt(50) = 4% of their spread at
most, the logits by less: root mean square over the tokens' logits, 10%.  A
token at the wrong place, or one that is not seen, changes them by all of it."""
import importlib.util
import os

import numpy as np
import pytest

from gpu_util import torch_dev

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder4.py")
    spec = importlib.util.spec_from_file_location("decoder4", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", [dict(), dict(hidden=256, heads=6, kv_heads=3, head_dim=96, inner=320, page=16)])
def test_decoding_continues_a_prompt(shape, kind):
    torch = torch_dev()
    lens, steps = [70, 1, 33], 40
    model = _example().Decoder(3, 200, vocab=512, dtype=getattr(torch, kind), **shape)
    rng = np.random.default_rng(7)
    text = [rng.integers(0, 512, n + steps).tolist() for n in lens]
    whole = model.prompt(text).float()
    ends = np.cumsum([n + steps for n in lens])
    begins = ends - np.array(lens) - steps
    model.prompt([t[:n] for t, n in zip(text, lens)])
    for i in range(steps):
        got = model.step(torch.tensor([t[n + i] for t, n in zip(text, lens)], device="cuda")).float()
        want = whole[torch.tensor(begins + np.array(lens) + i, device="cuda")]
        off = float((got - want).square().mean().sqrt() / want.square().mean().sqrt())
        assert off <= 0.1, f"step {i}: {off}"
    assert model.lens.tolist() == [n + steps for n in lens]


def test_the_captured_step_is_the_eager_one():
    torch = torch_dev()
    make = _example().Decoder
    lens = [40, 64, 5, 1]
    rng = np.random.default_rng(8)
    prompts = [rng.integers(0, 512, n).tolist() for n in lens]
    eager, graph = (make(4, 130, vocab=512) for _ in range(2))
    a, b = eager.prompt(prompts), graph.prompt(prompts)
    assert (a == b).all()
    replay = graph.capture()
    new = torch.tensor([3, 1, 4, 1], device="cuda")
    for i in range(30):
        x, y = eager.step(new), replay(new)
        torch.cuda.synchronize()
        assert (x == y).all(), f"step {i}"
        new = x.argmax(-1)
    assert eager.lens.tolist() == graph.lens.tolist() == [n + 30 for n in lens]


def test_tokens_past_the_capacity_are_refused():
    """On the host, before anything is launched: eagerly, captured, and for prompts."""
    torch = torch_dev()
    make = _example().Decoder
    model = make(2, 48, vocab=512, page=16)
    with pytest.raises(ValueError, match="holds 48"):
        model.prompt([[1] * 49, [1]])
    with pytest.raises(ValueError, match="2 sequences"):
        model.prompt([[1]])
    model.prompt([[1, 2, 3] * 15, [4]])
    new = torch.tensor([3, 4], device="cuda")
    model.step(new)
    replay = model.capture()
    for _ in range(2):
        assert bool(torch.isfinite(replay(new)).all())
    assert model.lens.tolist() == [48, 4]
    for call in (model.step, replay):
        with pytest.raises(ValueError, match="49 tokens"):
            call(new)
    assert model.lens.tolist() == [48, 4]

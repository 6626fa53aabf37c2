"""The decoder operators take tensors and streams of the current GPU alone: the
call is launched there, without order against another GPU's streams."""
import types

import pytest

import paper_2209_12982_amd as W
from paper_2209_12982_amd import binding


def _calls(make):
    """One call of each operator as (name, marshalled arguments); `make(shape, type)` gives the tensors."""
    import torch
    half, f32, i32, i64, u8 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8
    cache = tuple(make((2, 1, 16, w), u8) for w in (32, 2, 32, 2))
    q, k, cu = make((4, 2, 64), half), make((4, 1, 64), half), make((2,), i32)
    return [
        ("w4_matvec", (make((2, 64), half), make((8, 32), u8), make((8, 2), u8), make((2, 8), half), None, None)),
        ("kv4_append", (q, k, k, make((9, 64), f32), make((4,), i32), make((4,), i64), cache, make((4, 2, 64), half), None, None,
                        0, 0)),
        ("kv4_attention", (q, cache, make((4, 2), i32), make((4,), i32), make((4, 2, 64), half), 1.0, None)),
        ("prompt_attention", (q, k, k, cu, cu, 4, make((4, 2, 64), half), 1.0, True)),
    ]


def _module():
    try:
        return binding._marshal()
    except W.LibraryNotBuilt:
        pytest.skip("library not built")


@pytest.mark.parametrize("which", range(4))
def test_tensors_of_another_gpu_are_refused(which):
    """Tensors that say they are on GPU 1, without memory: refused before their addresses are asked for."""
    module = _module()
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    if torch.cuda.is_available():
        pytest.skip("needs no GPU, and no second one")
    with FakeTensorMode():
        name, args = _calls(lambda shape, t: torch.empty(shape, dtype=t, device="cuda:1"))[which]
        with pytest.raises(ValueError, match="current GPU"):
            getattr(module, name)(*args, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(4))
def test_calls_from_another_gpu_are_refused(which, monkeypatch):
    """The same with tensors of GPU 0 while another one is current, and with a stream of another one."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    name, args = _calls(lambda shape, t: torch.zeros(shape, dtype=t, device="cuda"))[which]
    call = getattr(W, name)
    call(*args)
    call(*args, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    with pytest.raises(ValueError, match="stream"):
        call(*args, stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    monkeypatch.setattr(binding, "_CURRENT", lambda: 1)
    monkeypatch.setattr(binding, "_CURRENT_STREAM", lambda device: 0)
    with pytest.raises(ValueError, match="current GPU"):
        call(*args)


@pytest.mark.gpu
def test_every_tensor_of_a_call_is_looked_at():
    """One tensor of a call at a time in host memory."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    for name, args in _calls(lambda shape, t: torch.zeros(shape, dtype=t, device="cuda")):
        for i, a in enumerate(args):
            for j in range(len(a) if isinstance(a, tuple) else 1):
                if not isinstance(a, (tuple, torch.Tensor)):
                    continue
                other = a[:j] + (a[j].cpu(),) + a[j + 1:] if isinstance(a, tuple) else a.cpu()
                with pytest.raises(ValueError, match="current GPU"):
                    getattr(W, name)(*args[:i], other, *args[i + 1:])

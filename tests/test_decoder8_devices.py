"""The 8-bit decoder operators take tensors and streams of the current GPU alone."""
import types

import pytest

import paper_2209_12982_amd as W
from paper_2209_12982_amd import binding


def _calls(make):
    """One call of each operator as (name, marshalled arguments); `make(shape, type)` gives the tensors."""
    import torch
    half, f32, i32, i8, u8 = torch.bfloat16, torch.float32, torch.int32, torch.int8, torch.uint8
    return [
        ("w8_quantize", (make((2, 64), half), make((2, 64), i8), make((2,), f32))),
        ("w8_matmul", (make((2, 64), i8), make((2,), f32), make((8, 64), i8), make((8,), f32), make((2, 8), half), make((8,), half),
                       make((64,), u8))),
        ("route_experts", (make((3, 4), f32), make((3, 2), i32), make((3, 2), f32), make((6,), i32), make((5,), i32), make((4,), f32),
                           0, 1, 1, 1, True, 1.0, make((1,), i32), make((256,), u8))),
        ("w8_experts_matmul", (make((3, 64), i8), make((3,), f32), make((4, 8, 64), i8), make((4, 8), f32), make((6,), i32),
                               make((5,), i32), make((3, 8), half), make((3, 2), i32), make((3, 2), f32), make((1024,), u8))),
    ]


@pytest.mark.parametrize("which", range(4))
def test_tensors_of_another_gpu_are_refused(which):
    """Tensors that say they are on GPU 1, without memory: refused before their addresses are asked for."""
    try:
        module = binding._marshal()
    except W.LibraryNotBuilt:
        pytest.skip("library not built")
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    if torch.cuda.is_available():
        pytest.skip("needs no GPU, and no second one")
    with FakeTensorMode():
        name, args = _calls(lambda shape, t: torch.empty(shape, dtype=t, device="cuda:1"))[which]
        with pytest.raises(ValueError, match="current GPU"):
            getattr(module, name)(*args, 0, 0)
        with pytest.raises(TypeError):
            getattr(module, name)(*args, 0)


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
            if isinstance(a, torch.Tensor):
                with pytest.raises(ValueError, match="current GPU"):
                    getattr(W, name)(*args[:i], a.cpu(), *args[i + 1:])

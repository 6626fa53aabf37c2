"""What a build needs: libwinof4.so hipcc alone; torch and a host compiler only
the decoder operators' Python binding."""
import ctypes
import os
import sys

import pytest

from paper_2209_12982_amd import build as B


def _build(tmp_path, monkeypatch):
    """A build of one source into a folder of its own."""
    try:
        B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    monkeypatch.setattr(B, "PKG", str(tmp_path))
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libwinof4.so"))
    monkeypatch.setattr(B, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(B, "SOURCES", ["w4_quantize.cpp"])
    return B.build()


@pytest.mark.parametrize("missing", ["torch", "g++"])
def test_the_library_needs_hipcc_alone(missing, tmp_path, monkeypatch, capsys):
    if missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setattr(B, "marshal_commands", lambda out: [["a-compiler-that-is-not-there", "-o", out]])
    lib = _build(tmp_path, monkeypatch)
    assert hasattr(ctypes.CDLL(lib), "w4_quantize_weights")
    assert not os.path.exists(B.MARSHAL) and "_marshal.so is not built" in capsys.readouterr().err


def test_sources_that_do_not_compile_fail_the_build(tmp_path, monkeypatch):
    monkeypatch.setattr(B, "marshal_commands", lambda out: [["false", "-o", out]])
    with pytest.raises(RuntimeError, match="marshal"):
        _build(tmp_path, monkeypatch)

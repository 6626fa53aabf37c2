"""Which kernels a call of the library launches, asked on the host: the call runs
in a process of its own whose launches are written down (launch_recorder.cpp)
and not made.  Addresses are never read."""
import json
import os
import re
import subprocess
import sys
import tempfile

import pytest

import paper_2209_12982_amd as W

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ADDRESS = 1 << 20           # aligned, and nobody's

_CHILD = """
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
sys.modules["torch"] = None         # the library by itself
recorder.launches_taken.restype = recorder.kernels_known.restype = ctypes.c_char_p
import paper_2209_12982_amd as W
lib = W.load_library()
out = []
for name, args, fail in json.load(sys.stdin):
    recorder.launches_taken(fail)
    status = getattr(lib, name)(*args)
    out.append([status, recorder.launches_taken(-1).decode()])
print(json.dumps([recorder.kernels_known().decode(), out]))
"""


def _plain(kernel):
    return re.sub(r"\bw8::|^void |\(.*\)$", "", kernel.replace("(anonymous namespace)::", ""))


def _ask(calls):
    try:
        W.load_library()
    except W.LibraryNotBuilt:
        pytest.skip("library not built")
    with tempfile.TemporaryDirectory() as folder:
        recorder = os.path.join(folder, "recorder.so")
        try:
            subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", recorder, os.path.join(HERE, "launch_recorder.cpp")],
                           check=True)
        except FileNotFoundError:
            pytest.skip("no host compiler")
        r = subprocess.run([sys.executable, "-c", _CHILD, recorder], input=json.dumps(calls), capture_output=True, text=True, cwd=ROOT,
                           timeout=300)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def kernels():
    """The names of all kernels that the library holds."""
    return [_plain(line) for line in _ask([])[0].splitlines()]


def launches(calls):
    """[(name, arguments, number of the launch that fails or -1)] -> [(status, [dict of kernel, grid, threads, shared])]."""
    out = []
    for status, text in _ask(calls)[1]:
        made = []
        for line in text.splitlines():
            grid, threads, shared, kernel = line.split("|", 3)
            made.append(dict(kernel=_plain(kernel), grid=[int(v) for v in grid.split()], threads=int(threads), shared=int(shared)))
        out.append((status, made))
    return out

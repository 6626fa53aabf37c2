"""What the 8-bit decoder operators launch, asked on the host without a GPU."""
import os
import subprocess

import pytest

from paper_2209_12982_amd import build as B

import decoder8_sizes as sizes
from launch_util import ADDRESS as P
from launch_util import kernels, launches


@pytest.mark.parametrize("fail", [0, 1])
def test_launches_that_fail_are_reported(fail):
    """The products and their weighted sums are two launches: whichever fails, the call says so, and nothing follows a failure."""
    args = [P, 64, P, 2, P, P, P, P, 4, 3, P, P, 2, P, 8, 8, 64, 0, P, 128, None]
    (good, both), (status, made) = launches([("w8_experts_matmul", args, -1), ("w8_experts_matmul", args, fail)])
    assert good == 0 and [m["kernel"].split("<")[0] for m in both] == ["w8_rows_kernel", "w8_combine_kernel"]
    assert status == -6 and made == both[:fail + 1]


def matmul(m, n, k, x_stride=None, room=1 << 40):
    return ("w8_matmul", [P, k if x_stride is None else x_stride, P, P, P, None, P, n, m, n, k, 0, P, room, None], -1)


def test_far_rows_that_a_launch_does_not_hold_are_refused():
    """Rows of x 2^25 bytes apart take tiles of 64 x 128, of which there are twice as many as of 128 x 128."""
    outs = 1 << 24
    calls = [matmul(rows, outs, 16, 1 << 25) for rows in (4096, 3969, 3968)]
    assert [status for status, made in launches(calls)] == [-2, -2, 0]


def test_grids_that_are_accepted_fit_a_launch():
    """A launch counts its threads in 32 bits, in each direction."""
    sizes = [(m, n, k) for m in (1, 30, 70, 1000, 5000, 40000, 1 << 20) for n in (1, 300, 4096, 1 << 17, 1 << 24) for k in (16, 1040, 65536)]
    calls = [matmul(m, n, k, stride) for m, n, k in sizes for stride in (k, 1 << 27)]
    done = launches(calls)
    assert sum(status == 0 for status, made in done) > 100
    for call, (status, made) in zip(calls, done):
        assert status in (0, -2) and bool(made) == (status == 0), call
        for m in made:
            assert m["grid"][0] * m["threads"] < 2 ** 32 and max(m["grid"][1:]) < 2 ** 16, (call, m)


def test_few_rows_fall_to_one_workgroup_each(tmp_path):
    """Up to 32 rows by the kernel for few: the sets that its workgroups take, over the grid that is launched, hold each row once."""
    try:
        hipcc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    sizes = [(m, n, k) for m in range(1, 33) for n, k in ((1407, 768), (8771, 112), (96, 16))]
    grids = set()
    for (m, n, k), (status, made) in zip(sizes, launches([matmul(*s) for s in sizes])):
        if made[0]["kernel"].startswith("w8_rows_kernel"):
            grids.add((m, made[0]["grid"][1]))
    assert {m for m, sets in grids} == set(range(1, 33))
    source = tmp_path / "sets.hip"
    source.write_text("""
#include "w8_rows.h"
constexpr bool once(int m, int sets) {
    for (int row = 0; row < m; ++row) {
        int times = 0;
        for (int s = 0; s < sets; ++s) times += w8::rows_of_set(s, 16, m).begin <= row && row < w8::rows_of_set(s, 16, m).end;
        if (times != 1) return false;
    }
    return w8::rows_of_set(sets - 1, 16, m).end == m;
}
""" + "".join(f"static_assert(once({m}, {sets}), \"{m} rows\");\n" for m, sets in sorted(grids)))
    r = subprocess.run([hipcc, "-std=c++17", "-fsyntax-only", "--offload-host-only", "-I", B.CSRC, "-I", os.path.join(B.ROOT, "include"),
                        str(source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_rows_that_are_not_there_are_not_far():
    """Fewer rows than a tile: how far the last of them lies decides, and the stride of a single one does not count."""
    sizes = [(m, n, k) for m in (1, 2, 5, 33) for n in (64, 5000) for k in (2064, 16384, 65536)]
    near, far = [], []
    for m, n, k in sizes:
        apart = ((1 << 32) - 1 - k) // (m - 1) // 16 * 16 if m > 1 else 1 << 62
        near.append(matmul(m, n, k))
        far.append(matmul(m, n, k, apart))
    plain = launches(near)
    assert any("w8_tiles" in made[0]["kernel"] for status, made in plain)
    assert launches(far) == plain


def experts(tokens, outs_of, top, n, k, weighted=False, apart=None):
    routes = tokens * top
    return ("w8_experts_matmul", [P, k if apart is None else apart, P, tokens, P, P, P, P, routes, outs_of, P if weighted else None,
                                  P if weighted else None, top, P, n, n, k, 0, P, 1 << 45, None], -1)


def route(tokens, of, top, kind=0):
    return ("route_experts", [P, of, None, tokens, of, top, 0, 1, 1, 1, 1, 1.0, None, P, P, P, P, kind, P, 1 << 40, None], -1)


def test_other_grids_fit_a_launch():
    calls = [experts(t, e, top, n, k, weighted) for t in (1, 100, 5000, 1 << 20) for e in (1, 60, 1024) for top in (1, 4)
             for n in (1, 4096, 1 << 20) for k in (16, 65536) for weighted in (False, True)]
    calls += [route(t, e, top) for t in (1, 33, 5000, 1 << 17, 1 << 22) for e in (1, 60, 256, 1024) for top in (1, 32) if top <= e]
    calls += [("w8_quantize", [P, k, P, P, m, k, 0, None], -1) for m in (1, 1 << 20, (1 << 24) - 1) for k in (16, 1 << 20)]
    done = launches(calls)
    assert sum(status == 0 for status, made in done) > 150
    for call, (status, made) in zip(calls, done):
        assert status in (0, -2) and bool(made) == (status == 0), call
        for m in made:
            assert m["grid"][0] * m["threads"] < 2 ** 32 and max(m["grid"][1:]) < 2 ** 16 and m["shared"] <= 160 << 10, (call, m)


def second(made):
    if len(made) > 1 and "combine" not in made[1]["kernel"]:
        return made[1]["kernel"].split("_")[1]
    return None


def test_sizes_take_their_kernels():
    """The table of sizes that the GPU tests run, kernel by kernel."""
    for table, call in ((sizes.MATMUL, matmul), (sizes.EXPERTS, experts)):
        listed = [(key, s) for key, many in table.items() for s in many]
        for (key, s), (status, made) in zip(listed, launches([call(*s) for key, s in listed])):
            few = call is experts and "rows" in made[0]["kernel"] and made[0]["grid"][1] < s[1]
            assert (sizes.name_of(made[0]["kernel"]), "few" if few else second(made)) == key and status == 0, (s, made)
    far = [matmul(*s) for s in sizes.MATMUL_FAR] + [experts(*s[:5], apart=s[5]) for s in sizes.EXPERTS_FAR]
    for call, (status, made) in zip(far, launches(far)):
        assert status == 0 and made[0]["kernel"].endswith("true>"), (call, made)
    near = [matmul(*s) for s in sizes.MATMUL_NEAR] + [experts(*s[:5], apart=s[5]) for s in sizes.EXPERTS_NEAR]
    for call, (status, made) in zip(near, launches(near)):
        assert status == 0 and made[0]["kernel"].endswith("false>") and "tiles" in made[0]["kernel"], (call, made)
    listed = [(key, s) for key, many in sizes.ROUTE.items() for s in many]
    for (key, s), (status, made) in zip(listed, launches([route(*s) for key, s in listed])):
        assert status == 0 and tuple(m["kernel"].replace(m["kernel"][m["kernel"].find("<"):], "") if "experts" in m["kernel"]
                                     else m["kernel"] for m in made) == key, (s, made)


def test_every_kernel_has_sizes():
    """What the table's calls launch, in either type, is every kernel of these operators that the library holds."""
    calls = [call(*s) for table, call in ((sizes.MATMUL, matmul), (sizes.EXPERTS, experts)) for many in table.values() for s in many]
    calls += [matmul(*s) for s in sizes.MATMUL_FAR] + [experts(*s[:5], apart=s[5]) for s in sizes.EXPERTS_FAR]
    calls += [experts(*s, weighted=True) for s in sizes.EXPERTS["32x32", None]]
    calls += [("w8_quantize", [P, k, P, P, 3, k, 0, None], -1) for k in (4096, 16384, 16400)]
    other = [(name, args[:at] + [1] + args[at + 1:], -1) for name, args, _ in calls
             for at in [{"w8_matmul": 11, "w8_experts_matmul": 17, "w8_quantize": 6}[name]]]
    calls += other + [route(*s, kind=kind) for many in sizes.ROUTE.values() for s in many for kind in (0, 1, 2)]
    launched = {m["kernel"] for status, made in launches(calls) for m in made}
    held = {k for k in kernels() if k.startswith(("w8_", "route_"))}
    assert len(held) > 50 and launched == held, (sorted(held - launched), sorted(launched - held))


@pytest.mark.parametrize("level", ["-O1", "-O2"])
def test_tiles_compile_at_other_levels(tmp_path, level):
    """The assembly in the copies gets the registers that it names, whatever the optimizer leaves of the code around it."""
    try:
        hipcc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    source = tmp_path / "tiles.hip"
    source.write_text("""
#include "w8_tiles.h"
template __global__ void w8::w8_tiles_kernel<WINO_BF16, w8::Tile256x256, false>(w8::Args, int, int);
template __global__ void w8::w8_tiles_kernel<WINO_FP16, w8::Tile64x64, true>(w8::Args, int, int);
template __global__ void w8::w8_tiles_kernel<WINO_FP16, w8::Tile64x128, true, true>(w8::Args, int, int);
""")
    flags = [level if f == "-O3" else f for f in B.HIP_FLAGS]
    r = subprocess.run([hipcc, *flags, "--offload-device-only", "-I", B.CSRC, "-I", os.path.join(B.ROOT, "include"), "-c", str(source),
                        "-o", str(tmp_path / "tiles.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

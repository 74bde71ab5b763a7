"""Launch shapes of the gated recurrence over ranges of sizes, on the CPU, and that the built library has kernels for
these shapes and for no others."""
import ctypes
import os
import re
import subprocess

import pytest

pytest.importorskip("msgpack")
from test_kernel_resources import _code_objects, _kernels  # noqa: E402

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_15976_amd", "csrc")

HARNESS = r"""
#include "lbscan_gated_plan.h"
extern "C" void shape(long rows, int seqlen, int dtype, int* out)
{
    const lbscan::GatedShape s = lbscan::gated_shape_of(rows, seqlen, dtype);
    const int v[] = {s.lanes, s.waves, s.ntiles, s.nseg, s.seg_tiles};
    for (int k = 0; k < 5; ++k) out[k] = v[k];
}
"""


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    d = tmp_path_factory.mktemp("gated_plan")
    src, lib = d / "plan.cpp", d / "plan.so"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(lib), str(src)], check=True)
    f = ctypes.CDLL(str(lib)).shape
    f.argtypes = [ctypes.c_long, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]

    def call(rows, seqlen, dtype):
        out = (ctypes.c_int * 5)()
        f(rows, seqlen, dtype, out)
        return tuple(out)

    return call


ROWS = [1, 2, 3, 7, 16, 40, 95, 96, 97, 128, 129, 255, 256, 257, 300, 512, 513, 700, 1024, 1025, 1500, 2048, 2049, 4096, 50000,
        (1 << 31) - 1]
LENGTHS = sorted({n * 64 * v + d for n in (1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 16, 17, 33, 100, 4000) for v in (4, 8) for d in (-1, 0, 1)}
                 | {1, 2, 7, 8, 9, 31, 32, 33, 64, 65, 100, 128, 197, 1 << 28, (1 << 28) - 1})


def family(s):
    """What a kernel is compiled for: lanes, waves, several tiles; a lane a row: None."""
    lanes, waves, ntiles, _, _ = s
    return None if lanes == 1 else (lanes, waves, ntiles > 1)


def test_shapes_cover_the_row(shape):
    for dtype in (0, 1):
        v = 4 if dtype == 0 else 8
        for rows in ROWS:
            for L in LENGTHS:
                s = lanes, waves, ntiles, nseg, seg_tiles = shape(rows, L, dtype)
                if L < 8:
                    assert s == (1, 1, 1, 1, 1)
                    continue
                tile = lanes * waves * v
                assert lanes in (8, 16, 32, 64) and waves in (1, 2, 4, 8, 16)
                assert lanes == 64 or (waves == 1 and ntiles == 1)
                assert (ntiles - 1) * tile < L <= ntiles * tile and ntiles * tile < 1 << 31
                assert 1 <= nseg <= 64 and (nseg - 1) * seg_tiles < ntiles <= nseg * seg_tiles
                # the kernels for cut rows are those of sixteen waves
                assert nseg == 1 or (waves == 16 and ntiles > 3 and rows <= 96), (rows, L, dtype, s)


def kernel_families():
    """Template arguments of the library's gated kernels, by forward and backward: (lanes, waves, several tiles, starts,
    summary)."""
    from paper_2506_15976_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_15976_amd import build
        build.build(force=True, verbose=False)
    with open(binding.LIB_PATH, "rb") as f:
        lib = f.read()
    found = {"fwd": set(), "bwd": set()}
    for elf in _code_objects(lib):
        for k in _kernels(elf):
            m = re.search(r"gated_(fwd|bwd)_kernelILi(\d+)ELi(\d+)ELb([01])ELb([01])ELb([01])E", k[".name"])
            if m:
                found[m[1]].add((int(m[2]), int(m[3]), m[4] == "1", m[5] == "1", m[6] == "1"))
    return found


def test_kernels_are_those_that_calls_reach(shape):
    reached, cut = set(), set()
    for dtype in (0, 1):
        for rows in ROWS:
            for L in LENGTHS:
                s = shape(rows, L, dtype)
                if family(s):
                    reached.add(family(s))
                    if s[3] > 1:
                        cut.add(family(s))
    want = {f + (starts, False) for f in reached for starts in (False, True)}
    want |= {f + (starts, True) for f in cut for starts in (False, True)}
    found = kernel_families()
    assert found["fwd"] == want and found["bwd"] == want

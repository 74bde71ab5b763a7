"""Which way the calls of loss_branches take, by the plan's own functions compiled for the host; no GPU."""
import ctypes
import os
import subprocess

import pytest

from loss_branches import CALLS, live

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_15976_amd", "csrc")

SOURCE = """
#include "lbscan_loss_plan.h"
using namespace lbscan;
// the choice of the parts of dweight's sums, as a wave makes it: the first of the smallest time
static int parts(const LossPlan& p, int dim, int live, int count)
{
    if (!p.share_rows) return 1;
    const long tiles = loss_ceil(count, loss_tokens(0, 2)), m = loss_ceil(p.dimp, kLossTile), most = p.share_rows / (tiles * loss_tokens(0, 2));
    const int steps = loss_ceil32(live, 32);
    int best = 1;
    for (int s = 2; s <= 64; ++s)
        if (s <= loss_most_splits(256) && loss_split_fits(steps, s, most) &&
            loss_split_time(m * tiles, steps, s, 256, 2) < loss_split_time(m * tiles, steps, best, 256, 2)) best = s;
    return best;
}
extern "C" void ways(long tokens, int vocab, int dim, int live, int* out)
{
    const LossPlan p = loss_plan_of(tokens, vocab, dim, 2, true, true, true, true, 0);
    out[0] = p.pieces;
    out[1] = parts(p, dim, live, p.piece);
    out[2] = parts(p, dim, live, vocab - (p.pieces - 1) * p.piece);
    out[3] = p.loose;
    out[4] = p.copy_weight;
}
"""


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    at = tmp_path_factory.mktemp("ways")
    (at / "ways.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-I", CSRC, str(at / "ways.cpp"), "-o", str(at / "ways.so")], check=True)
    lib = ctypes.CDLL(str(at / "ways.so"))

    def call(tokens, vocab, dim, n):
        out = (ctypes.c_int * 5)()
        lib.ways(ctypes.c_long(tokens), vocab, dim, n, out)
        return list(out)
    return call


@pytest.mark.parametrize("T,V,D,ignored,before,last,rows", CALLS)
def test_the_way_of_each_call(ways, T, V, D, ignored, before, last, rows):
    pieces, parts_before, parts_last, loose, copied = ways(T, V, D, len(live(T, ignored)))
    name = lambda parts: "cut" if parts > 1 else "whole"  # noqa: E731
    assert name(parts_last) == last and rows == ("loose" if loose else "copied" if copied else "in place")
    assert (before is None) == (pieces == 1) and (before is None or name(parts_before) == before)


def test_every_way_is_taken():
    assert {c[5] for c in CALLS} | {c[4] for c in CALLS} >= {"cut", "whole"} and {c[6] for c in CALLS} == {"in place", "loose", "copied"}
    assert all(sum(c[0] <= 64 and c[6] == rows for c in CALLS) >= 2 for rows in ("in place", "loose"))

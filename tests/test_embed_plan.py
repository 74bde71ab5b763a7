"""The mask of groups in the embedding gradient's sort, for every number of groups that a wave may have, on the CPU."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_15976_amd", "csrc")


@pytest.fixture(scope="module")
def span(tmp_path_factory):
    d = tmp_path_factory.mktemp("embed_plan")
    src, lib = d / "plan.cpp", d / "plan.so"
    src.write_text('#include "lbscan_embed_plan.h"\nextern "C" int span(long groups) { return lbscan::sort_span_log2(groups); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(lib), str(src)], check=True)
    f = ctypes.CDLL(str(lib)).span
    f.argtypes = [ctypes.c_long]
    return f


def test_every_group_has_a_bit(span):
    # 2^31 tokens, a wave of eight: 2^22 groups
    numbers = set(range(0, 70000)) | {(1 << k) + d for k in range(17, 23) for d in (-1, 0, 1)}
    for groups in numbers:
        k = span(groups)
        assert 0 <= k < 32
        if groups:
            assert (groups - 1) >> k <= 63, groups          # a shift of 64 bits by more than 63 is undefined
        # no coarser than needed: a bit too coarse looks at groups again that have nothing
        assert k == 0 or (groups - 1) >> (k - 1) > 63, groups

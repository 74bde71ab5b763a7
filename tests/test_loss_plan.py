"""The plan of the loss (sizes, pieces, scratch) over ranges of sizes: compiled for the host, no GPU."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_15976_amd", "csrc")
NUMBERS = ("dimp", "rows", "few", "loose", "copy_weight", "piece", "pieces", "part_room", "acc_rows", "share_rows")
FIELDS = ("choice", "counts", "rank", "order", "targets", "lse2", "down", "both", "own", "part", "x", "w", "g", "acc", "share", "hot", "rest",
          "rest_rows", "list", "slot", "sort", "total")


SORT = 12345


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    src = at / "plan.cpp"
    src.write_text('#include "lbscan_loss_plan.h"\n'
                   'extern "C" void plan(long t, int v, int d, int e, int al, int b, int dx, int dw, long sort, long* o) {\n'
                   '  const lbscan::LossPlan p = lbscan::loss_plan_of(t, v, d, e, al, b, dx, dw, sort);\n'
                   f'  const long n[] = {{{", ".join("p." + f for f in NUMBERS)}}};\n'
                   f'  for (int i = 0; i < {len(NUMBERS)}; ++i) o[i] = n[i];\n'
                   f'  const size_t at[] = {{{", ".join("p." + f for f in FIELDS)}}};\n'
                   f'  for (int i = 0; i < {len(FIELDS)}; ++i) o[{len(NUMBERS)} + i] = at[i];\n}}\n')
    so = at / "plan.so"
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))

    def call(tokens, vocab, dim, element, aligned, backward, dx=1, dw=1):
        out = (ctypes.c_long * (len(NUMBERS) + len(FIELDS)))()
        lib.plan(ctypes.c_long(tokens), vocab, dim, element, aligned, backward, dx, dw, ctypes.c_long(SORT), out)
        return dict(zip(NUMBERS + FIELDS, out))
    return call


def test_sizes_and_scratch(plan):
    rng = random.Random(1)
    log = lambda lo, hi: int(round(2 ** rng.uniform(lo, hi)))  # noqa: E731
    for _ in range(3000):
        T, V, D, e = log(0, 24), log(0, 20), log(0, 16), rng.choice([2, 4])
        aligned, backward, dx, dw = (rng.randrange(2) for _ in range(4))
        p = plan(T, V, D, e, aligned, backward, dx, dw)
        tile = 64 if p["few"] else 256 if e == 2 else 128
        whole = 256 // e if p["loose"] else 64 // e
        assert p["dimp"] % whole == 0 and 0 <= p["dimp"] - D < whole
        assert p["rows"] % tile == 0 and 0 <= p["rows"] - T < tile
        odd = not aligned or D % (64 // e) != 0
        assert p["loose"] == int(odd and p["few"] and D * e >= 16) and p["copy_weight"] == int(odd and not p["loose"])
        # the pieces cover the vocabulary, none is empty, and the offsets of a block's lines fit 32 bits
        assert p["piece"] % 256 == 0 and (p["pieces"] - 1) * p["piece"] < V <= p["pieces"] * p["piece"]
        assert p["piece"] * e * 256 < 1 << 32 and p["dimp"] * e * 256 < 1 << 32
        assert p["rows"] * p["piece"] * e <= max(1 << 30, p["rows"] * 256 * e)
        # room for one part of every sum at the least
        assert backward or p["part_room"] >= p["rows"]
        assert not (backward and dx) or p["acc_rows"] >= p["rows"]
        used = {"choice": 32, "counts": 4 * -(-T // 1024), "rank": 4 * T, "order": 4 * p["rows"], "targets": 4 * p["rows"],
                "x": p["rows"] * p["dimp"] * e}
        if p["copy_weight"]:
            used["w"] = V * p["dimp"] * e
        if backward:
            used.update({k: 4 * p["rows"] for k in ("lse2", "down", "both")}, g=p["rows"] * p["piece"] * e)
            if e == 2:
                used.update(hot=4 * p["rows"], rest=4 * p["rows"])
                if dw:
                    used.update(rest_rows=2 * p["rows"] * p["dimp"], list=2 * p["rows"] * p["dimp"], slot=4 * V, sort=SORT)
            if dx:
                used["acc"] = 4 * p["acc_rows"] * p["dimp"]
            if dw and p["share_rows"]:
                used["share"] = 4 * p["share_rows"] * p["dimp"]
        else:
            used.update(own=4 * p["rows"], part=8 * p["part_room"])
        at = sorted((p[k], k) for k in used)
        for (a, k), (b, _) in zip(at, at[1:] + [(p["total"], "")]):
            assert a % 256 == 0 and a + used[k] <= b, (k, T, V, D)


def test_nothing_to_do(plan):
    for T, V in ((0, 5), (5, 0)):
        assert plan(T, V, 64, 2, 1, 1)["total"] == 0


def test_a_backward_call_that_wants_less_fits_the_room_for_both(plan):
    rng = random.Random(2)
    for _ in range(500):
        T, V, D = rng.randrange(1, 5000), rng.randrange(1, 200000), rng.randrange(1, 3000)
        whole = plan(T, V, D, 2, 1, 1)["total"]
        assert plan(T, V, D, 2, 1, 1, 1, 0)["total"] <= whole and plan(T, V, D, 2, 1, 1, 0, 1)["total"] <= whole

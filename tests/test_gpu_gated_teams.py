"""The gated recurrence in every team that its launch rule has for rows of several tiles, both ways, packed and not: what is
carried from tile to tile, and the states kept at their starts."""
import pytest

import sequence_reference as ref
from sequence_util import GATED, TYPES, close, to_numpy
from test_gated_plan import shape  # noqa: F401  (a fixture)

# type, waves of a team, tiles: batch, dim, tokens
SIZES = [("fp32", 1, 5, 21, 100, 1200), ("bf16", 1, 5, 21, 100, 2300), ("fp32", 2, 3, 11, 100, 1200), ("bf16", 2, 3, 11, 100, 2300),
         ("fp32", 4, 3, 6, 100, 2200), ("bf16", 4, 3, 6, 100, 4400), ("fp32", 8, 3, 3, 100, 5000), ("bf16", 8, 3, 3, 100, 9000),
         ("fp32", 16, 3, 1, 100, 9001), ("bf16", 16, 2, 1, 100, 9001)]


def test_sizes_are_of_these_teams(shape):  # noqa: F811
    for dtype, waves, tiles, batch, dim, tokens in SIZES:
        assert shape(batch * dim, tokens, ("fp32", "bf16").index(dtype)) == (64, waves, tiles, 1, tiles)


@pytest.fixture(scope="module")
def lb():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


@pytest.mark.gpu
@pytest.mark.parametrize("starts", [False, True])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype,waves,tiles,batch,dim,tokens", SIZES)
def test_team(lb, dtype, waves, tiles, batch, dim, tokens, reverse, starts):
    import torch
    g = torch.Generator().manual_seed(tokens)
    t = {k: torch.randn(batch, dim, tokens, generator=g).to(TYPES[dtype]).cuda() for k in ("x", "gate_a", "gate_x")}
    open_gate = torch.empty(dim).uniform_(0.9, 0.999, generator=g)
    t["decay"] = torch.log(torch.expm1(-torch.log(open_gate) / 8)).cuda()
    t["h0"] = torch.randn(batch, dim, generator=g).cuda()
    if starts:
        t["starts"] = (torch.rand(batch, tokens, generator=g) < 4.0 / tokens).cuda()
    dout = torch.randn(batch, dim, tokens, generator=g).to(TYPES[dtype]).cuda()
    dhT = torch.randn(batch, dim, generator=g).cuda()
    n = {k: to_numpy(v) for k, v in t.items()}
    keys = dict(starts=n.get("starts"), reverse=reverse, h0=n["h0"])
    y, hT, _ = ref.gated_fwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], **keys)
    want = ref.gated_bwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], to_numpy(dout), dhT=to_numpy(dhT), **keys)
    saved = lb.lbscan_gated_saved_state(t["x"], reverse=reverse)
    assert saved.numel() == batch * dim * tiles
    got, gT = lb.lbscan_gated_fwd(**t, reverse=reverse, return_state=True, saved_state=saved)
    close(got, y, GATED[dtype], "y")
    close(gT, hT, GATED["fp32"], "hT")
    kept = lb.lbscan_gated_bwd(**t, dout=dout, dhT=dhT, reverse=reverse, saved_state=saved)
    for k, v in kept.items():
        close(v, want[k], GATED["fp32"] if k in ("ddecay", "dh0") else GATED[dtype], k)
    again = lb.lbscan_gated_bwd(**t, dout=dout, dhT=dhT, reverse=reverse)
    assert all(torch.equal(kept[k], again[k]) for k in kept)

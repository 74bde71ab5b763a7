"""The operators around the scan at random sizes, types and options against the 64-bit reference."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from sequence_util import GATED, NORM, TYPES, close, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def gated_tolerance(dtype, keep):
    """The derivation of sequence_util for states that remember longer: half open gates keep `keep` ** 0.5, so up to
    M = 2 / (1 - keep) tokens count; 8 u sqrt(M) of a state, five times that at the floor.  M there: 2000."""
    longest = (float(2 / (1 - keep.max())) / 2000) ** 0.5
    return tuple(max(1.0, longest) * v for v in GATED["fp32"]) if dtype == "fp32" else GATED["bf16"]


def size(rng, lo, hi):
    return int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))


@pytest.mark.parametrize("seed", range(24))
def test_gated(lb, seed):
    rng = np.random.default_rng(seed)
    L = size(rng, 2, 20000)
    B, D = size(rng, 1, 40), size(rng, 1, 400)
    while B * D * L > 3e6:
        B, D = (B + 1) // 2, (D + 1) // 2
        L = L if B * D > 1 else int(3e6)
    dtype, reverse = ("fp32", "bf16")[rng.integers(2)], bool(rng.integers(2))
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    t = {k: torch.randn(B, D, L, generator=g).to(dt).cuda() for k in ("x", "gate_a", "gate_x")}
    # open gates that keep 0.5 .. 0.9999 of the state: rows near one and others
    keep = torch.exp(-torch.exp(torch.empty(D).uniform_(np.log(1e-4), np.log(0.7), generator=g)))
    t["decay"] = torch.log(torch.expm1(-torch.log(keep) / 8)).cuda()
    if rng.integers(2):
        t["starts"] = (torch.rand(B, L, generator=g) < 2.0 / (1 + L ** 0.5)).cuda()
    if rng.integers(2):
        t["h0"] = torch.randn(B, D, generator=g).cuda()
    dout = torch.randn(B, D, L, generator=g).to(dt).cuda()
    n = {k: to_numpy(v) for k, v in t.items()}
    keys = dict(starts=n.get("starts"), reverse=reverse, h0=n.get("h0"))
    y, h, _ = ref.gated_fwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], **keys)
    want = ref.gated_bwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], to_numpy(dout), **keys)
    saved = lb.lbscan_gated_saved_state(t["x"], reverse=reverse)
    got, gT = lb.lbscan_gated_fwd(**t, reverse=reverse, return_state=True, saved_state=saved)
    where = f"{B} x {D} x {L} {dtype} "
    tol, exact = gated_tolerance(dtype, keep), gated_tolerance("fp32", keep)
    close(got, y, tol, where + "y")
    close(gT, h, exact, where + "hT")
    for k, v in lb.lbscan_gated_bwd(**t, dout=dout, reverse=reverse, saved_state=saved).items():
        close(v, want[k], exact if k in ("ddecay", "dh0") else tol, where + k)


@pytest.mark.parametrize("seed", range(24))
def test_norm(lb, seed):
    rng = np.random.default_rng(100 + seed)
    dim, rows = size(rng, 2, 16000), size(rng, 1, 20000)
    rows = max(1, min(rows, int(4e6) // dim))
    dtype, residual = ("fp32", "bf16")[rng.integers(2)], bool(rng.integers(2))
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, dim, generator=g) + 0.5).to(TYPES[dtype]).cuda()
    w, b = (1 + 0.3 * torch.randn(dim, generator=g)).cuda(), torch.randn(dim, generator=g).cuda()
    r = torch.randn(rows, dim, generator=g).cuda() if residual else None
    dout = torch.randn(rows, dim, generator=g).to(TYPES[dtype]).cuda()
    dsum = torch.randn(rows, dim, generator=g).cuda() if residual else None
    res = lb.lbscan_norm_fwd(x, w, b, residual=r, return_stats=True)
    total = res[1] if residual else None
    y, s, _, _ = ref.norm_fwd(to_numpy(x), to_numpy(w), to_numpy(b), None if r is None else to_numpy(r))
    where = f"{rows} x {dim} {dtype} "
    close(res[0], y, NORM[dtype], where + "y")
    want = ref.norm_bwd(to_numpy(x) if total is None else to_numpy(total), to_numpy(w), to_numpy(dout),
                        None if dsum is None else to_numpy(dsum))
    got = lb.lbscan_norm_bwd(None if residual else x, w, dout=dout, mean=res[-2], rstd=res[-1], total=total, dsum=dsum)
    if dim > 2:         # (two columns: the gradient is zero but for eps, and rounding is all of it)
        close(got["dx"], want["ds"], NORM[dtype], where + "dx")
    close(got["dweight"], want["dweight"], NORM["fp32"], where + "dweight")
    close(got["dbias"], want["dbias"], NORM["fp32"], where + "dbias")


@pytest.mark.parametrize("seed", range(24))
def test_embed(lb, seed):
    rng = np.random.default_rng(200 + seed)
    n, vocab, dim = size(rng, 1, 30000), size(rng, 1, 100000), size(rng, 1, 1500)
    n, vocab = max(1, min(n, int(4e6) // dim)), max(1, min(vocab, int(8e6) // dim))
    dtype = ("fp32", "bf16")[rng.integers(2)]
    g = torch.Generator().manual_seed(seed)
    ids = (torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * np.log(vocab + 1)) - 1).long().clamp(0, vocab - 1)
    if rng.integers(2):
        ids[torch.rand(n, generator=g) < 0.3] = -1
    dout = torch.randn(n, dim, generator=g).to(TYPES[dtype])
    ok = ids >= 0
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, ids[ok], dout.double()[ok]) * 0.7
    size_of = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, ids[ok], dout.double().abs()[ok]) * 0.7
    kind = torch.int32 if rng.integers(2) else torch.int64
    got = lb.lbscan_embed_bwd(ids.to(kind).cuda(), dout=dout.cuda(), vocab=vocab, scale=0.7).double().cpu()
    count = torch.bincount(ids[ok], minlength=vocab)[:, None].clamp(max=100)
    bound = (count + 2) * 2.0 ** -24 * size_of + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
    assert bool(((got - want).abs() <= bound).all()), f"{n} tokens of {vocab} x {dim} {dtype}"

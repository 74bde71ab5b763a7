"""Layer norm on the GPU against the 64-bit reference: every family of launch shapes, with and without the
residual stream, in place, constant rows, offsets, absent parameters."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from sequence_util import NORM, TYPES, close, off_by_one, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def make(rows, dim, dtype, residual, seed=0):
    g = torch.Generator().manual_seed(100 * seed + dim)
    t = dict(x=torch.randn(rows, dim, generator=g).to(TYPES[dtype]), weight=1 + 0.3 * torch.randn(dim, generator=g),
             bias=torch.randn(dim, generator=g))
    if residual:
        t["residual"] = 2 * torch.randn(rows, dim, generator=g) + 0.5
    dout = torch.randn(rows, dim, generator=g).to(TYPES[dtype])
    dsum = torch.randn(rows, dim, generator=g) if residual else None
    return {k: v.cuda() for k, v in t.items()}, dout.cuda(), None if dsum is None else dsum.cuda()


def check(lb, t, dout, dsum, dtype, eps=1e-5):
    n = {k: to_numpy(v) for k, v in t.items()}
    y, s, mean, rstd = ref.norm_fwd(n["x"], n.get("weight"), n.get("bias"), n.get("residual"), eps)
    res = lb.lbscan_norm_fwd(**t, eps=eps, return_stats=True)
    close(res[0], y, NORM[dtype], "y")
    close(res[-2], mean, (1e-4, 1e-6), "mean")         # (sums of signed values: their own floor)
    close(res[-1], rstd, NORM["fp32"], "rstd")
    total = res[1] if dsum is not None else None
    if total is not None:
        close(total, s, NORM["fp32"], "sum")
    want = ref.norm_bwd(s if total is None else to_numpy(total), n.get("weight"), to_numpy(dout),
                        None if dsum is None else to_numpy(dsum), eps)
    g = lb.lbscan_norm_bwd(t["x"] if total is None else None, t.get("weight"), dout=dout, mean=res[-2], rstd=res[-1],
                           with_bias="bias" in t, total=total, dsum=dsum)
    close(g["dx"], want["ds"], NORM[dtype], "dx")
    if total is not None:
        close(g["dresidual"], want["ds"], NORM["fp32"], "dresidual")
    for k in ("dweight", "dbias"):
        assert (g[k] is None) == (k[1:] not in t)
        if g[k] is not None:
            close(g[k], want[k], NORM["fp32"], k)


DIMS = [1, 2, 3, 7, 8, 9, 50, 64, 65, 127, 128, 255, 256, 257, 385, 512, 768, 1000, 1024, 1025, 2047, 2048, 2500, 4096,
        4100, 8191, 8192, 8193, 12288, 12289, 20000]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dim", DIMS)
def test_widths(lb, dim, residual, dtype):
    if dim == 1:                                     # a row of one value is its own mean: y is the bias
        t, _, _ = make(5, 1, dtype, residual)
        y = lb.lbscan_norm_fwd(**t)
        y = y[0] if residual else y
        assert torch.equal(y, t["bias"].to(y.dtype).expand(5, 1))
        return
    t, dout, dsum = make(5, dim, dtype, residual)
    check(lb, t, dout, dsum, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,dim", [(1, 768), (4, 64), (33, 40), (3001, 96), (9000, 385), (5000, 1030), (1500, 5000), (700, 12288)])
def test_rows(lb, rows, dim, residual, dtype):
    t, dout, dsum = make(rows, dim, dtype, residual, seed=1)
    check(lb, t, dout, dsum, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [24, 768])
def test_absent_parameters(lb, dim, dtype):
    for drop in (("weight",), ("bias",), ("weight", "bias")):
        for residual in (False, True):
            t, dout, dsum = make(6, dim, dtype, residual, seed=2)
            for k in drop:
                del t[k]
            check(lb, t, dout, dsum, dtype)
    t, dout, _ = make(6, dim, dtype, True, seed=2)
    # no gradient arrives at the sum
    res = lb.lbscan_norm_fwd(**t, return_stats=True)
    g = lb.lbscan_norm_bwd(None, t["weight"], dout=dout, mean=res[2], rstd=res[3], total=res[1])
    want = ref.norm_bwd(to_numpy(res[1]), to_numpy(t["weight"]), to_numpy(dout))
    close(g["dresidual"], want["ds"], NORM["fp32"], "dresidual")


@pytest.mark.parametrize("dim", [20, 777, 3000])
def test_offsets_and_constant_rows(lb, dim):
    """A mean far from zero costs no bits of the deviations; a constant row has none, and the bias is left."""
    t, dout, _ = make(4, dim, "fp32", False, seed=3)
    t["x"][0] += 4096.0
    t["x"][1] = 3.25
    t["x"][2] = 0.0
    x = to_numpy(t["x"])
    y = lb.lbscan_norm_fwd(**t)
    want = ref.norm_fwd(x, to_numpy(t["weight"]), to_numpy(t["bias"]))[0]
    # the mean is off by up to 2^-24 of itself, 2.4e-4 of a deviation of one
    assert np.abs(to_numpy(y)[0] - want[0]).max() < 2e-3
    assert torch.equal(y[1], t["bias"]) and torch.equal(y[2], t["bias"])
    close(y[3], want[3], NORM["fp32"], "y")
    res = lb.lbscan_norm_fwd(**t, eps=1e-5, return_stats=True)
    g = lb.lbscan_norm_bwd(t["x"], t["weight"], dout=dout, mean=res[1], rstd=res[2])
    assert all(bool(torch.isfinite(v).all()) for v in g.values() if v is not None)


def test_other_rows_stay_clean(lb):
    t, dout, _ = make(6, 130, "fp32", False, seed=4)
    clean = lb.lbscan_norm_fwd(**t)
    t["x"][2, 5] = float("nan")
    t["x"][4, 129] = float("inf")
    y = lb.lbscan_norm_fwd(**t)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[4]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [9, 100, 771, 2050, 12001, 12300])
def test_alignment_and_in_place(lb, dim, dtype):
    t, dout, dsum = make(7, dim, dtype, True, seed=5)
    y, s, mean, rstd = lb.lbscan_norm_fwd(**t, return_stats=True)
    moved = {k: off_by_one(v) for k, v in t.items()}
    ym, sm = lb.lbscan_norm_fwd(**moved, out=off_by_one(torch.zeros_like(y)))
    assert torch.equal(ym, y) and torch.equal(sm, s)
    a = lb.lbscan_norm_bwd(None, t["weight"], dout=dout, mean=mean, rstd=rstd, total=s, dsum=dsum)
    b = lb.lbscan_norm_bwd(None, moved["weight"], dout=off_by_one(dout), mean=off_by_one(mean), rstd=off_by_one(rstd),
                           total=off_by_one(s), dsum=off_by_one(dsum))
    assert all(torch.equal(a[k], b[k]) for k in a)
    # y over x, and through the C entry the sum over the residual
    import ctypes
    from paper_2506_15976_amd import binding
    x, r = t["x"].clone(), t["residual"].clone()
    args = lb.LbscanNormArgs(7, dim, int(dtype == "bf16"), 1e-5, x.data_ptr(), r.data_ptr(), t["weight"].data_ptr(),
                             t["bias"].data_ptr(), x.data_ptr(), r.data_ptr())
    assert lb.load().lbscan_norm_fwd(ctypes.byref(args), binding._stream(None)) == 0
    assert torch.equal(x, y) and torch.equal(r, s)


def test_shapes_and_empty(lb):
    x = torch.randn(2, 3, 5, 64, device="cuda")
    y = lb.lbscan_norm_fwd(x)
    assert torch.equal(y.view(-1, 64), lb.lbscan_norm_fwd(x.view(-1, 64)))
    assert lb.lbscan_norm_fwd(x[:0]).shape == (0, 3, 5, 64)
    assert lb.lbscan_norm_fwd(x[..., :0].contiguous()).shape == (2, 3, 5, 0)
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    g = lb.lbscan_norm_bwd(e, w, dout=e, mean=e[:, 0], rstd=e[:, 0])
    assert g["dx"].shape == (0, 64) and not g["dweight"].any() and not g["dbias"].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
def test_autograd(lb, residual, dtype):
    from paper_2506_15976_amd.autograd import layer_norm
    t, dout, dsum = make(30, 200, dtype, residual, seed=6)
    n = {k: to_numpy(v) for k, v in t.items()}
    leaves = [v.requires_grad_(True) for v in t.values()]
    out = layer_norm(**t)
    s = n["x"] + n["residual"] if residual else n["x"]
    want = ref.norm_bwd(s, n["weight"], to_numpy(dout), to_numpy(dsum) if residual else None)
    grads = torch.autograd.grad(out, leaves, (dout, dsum) if residual else dout)
    tol = NORM[dtype]
    close(grads[0], want["ds"], tol, "dx")
    close(grads[1], want["dweight"], NORM["fp32"], "dweight")
    close(grads[2], want["dbias"], NORM["fp32"], "dbias")
    if residual:
        close(grads[3], want["ds"], NORM["fp32"], "dresidual")
        # a loss on the sum alone: the norm passes nothing on
        _, total = layer_norm(**t)
        dx, dr = torch.autograd.grad(total, [t["x"], t["residual"]], dsum)
        assert torch.equal(dr, dsum) and torch.equal(dx, dsum.to(dx.dtype))


def test_same_bits_and_streams(lb):
    t, dout, dsum = make(5000, 300, "bf16", True, seed=7)
    y, s, mean, rstd = lb.lbscan_norm_fwd(**t, return_stats=True)
    call = dict(dout=dout, mean=mean, rstd=rstd, total=s, dsum=dsum)
    a = lb.lbscan_norm_bwd(None, t["weight"], **call)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    b = lb.lbscan_norm_bwd(None, t["weight"], **call, stream=stream)
    ys, ss = lb.lbscan_norm_fwd(**t, stream=stream)
    stream.synchronize()
    assert all(torch.equal(a[k], b[k]) for k in a)
    assert torch.equal(ys, y) and torch.equal(ss, s)

"""Softmax cross entropy over a vocabulary on the GPU against 64 bits: sizes around every tile and piece, ignored tokens, what
they hold, scales, absent gradients, peaked and flat logits, alignment, empty sizes, autograd, graphs, streams.

Tolerances, with u = 2^-24 and size = sum_d |scale x_td w_vd|, the sum of a logit's terms' sizes:
 * a logit is off by at most d = (2 sqrt(dim) + 8) u size: products are exact (bf16) or rounded once, the sum's dim roundings
   add up as sqrt(dim), twice that for the largest of many; scale and log2(e) are a rounding each.  lse is off by as much as the
   worst logit and 8 u of itself, loss by twice that.
 * G: its exponent is off by 2 d and 8 u |lse|, so G by that factor of its two terms' sizes; as bf16 it is rounded by at most
   2^-8 of it.  dx and dweight: that of the sum of their terms' sizes (whatever their signs), 2 sqrt(terms) u of the sum, and
   their own rounding, 2^-8 in bf16.  A bound for every element; their mean has to be below 2^-7 of rms (bf16: two
   independent roundings of 2^-8) or the relative bound above (fp32).
"""
import math

import pytest
import torch

import model_reference as ref
from model_util import HALF_STEP, TYPES, generator, guarded
from sequence_util import off_by_one

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def inputs(T, V, D, dtype, *, seed=0, ignored=0.0, peak=2.0):
    g = generator(seed)
    x = torch.randn(T, D, device="cuda", generator=g).to(dtype)
    w = (torch.randn(V, D, device="cuda", generator=g) * (peak / math.sqrt(D))).to(dtype)
    y = torch.randint(0, max(V, 1), (T,), device="cuda", generator=g)
    if ignored:
        y = torch.where(torch.rand(T, device="cuda", generator=g) < ignored, -100, y)
    return x, w, y


def check(lb, x, w, y, *, scale=1.0, dloss=None, dlse=None, gradients=True):
    T, D = x.shape
    V = w.shape[0]
    X, W, Y = x.double().cpu(), w.double().cpu(), y.cpu().long()
    live = (Y >= 0) & (Y < V)
    X = torch.where(live[:, None], X, torch.zeros(()).double())
    want_loss, want_lse = ref.loss(X, W, Y, scale=scale)
    size = float((abs(scale) * X.abs() @ W.abs().T).max()) if T * V else 0.0
    d = (2 * math.sqrt(D) + 8) * U * size
    loss, lse = lb.lbscan_loss_fwd(x, w, y, scale=scale)
    top = float(want_lse.abs().max()) if T else 0.0
    for name, got, want, times in (("lse", lse, want_lse, 1), ("loss", loss, want_loss, 2)):
        assert got.dtype == torch.float32 and got.shape == y.shape
        worst = float((got.double().cpu() - want).abs().max()) if T else 0.0
        assert worst <= times * (d + 8 * U * top) + 1e-12, f"{name}: {worst:.2e}, expected {times * (d + 8 * U * top):.2e}"
    assert not loss.cpu()[~live].any() and not lse.cpu()[~live].any()
    if not gradients:
        return
    g = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=dloss, dlse=dlse, scale=scale)
    down = (torch.zeros(T) if dloss is None else dloss.cpu()).double() * live
    both = down + (0 if dlse is None else dlse.cpu().double() * live)
    p = torch.softmax(scale * X @ W.T, 1) if V else torch.zeros(T, 0).double()
    hot = torch.zeros(T, V).double()
    hot[live, Y[live]] = 1.0
    G, sizes = both[:, None] * p - down[:, None] * hot, both.abs()[:, None] * p + down.abs()[:, None] * hot
    narrow = x.dtype == torch.bfloat16
    relative = 2 * d + 8 * U * (1 + top)
    for name, got, want, terms, count in (("dx", g["dx"], scale * G @ W, abs(scale) * sizes @ W.abs(), V),
                                          ("dweight", g["dweight"], scale * G.T @ X, abs(scale) * sizes.T @ X.abs(), T)):
        assert got.dtype == x.dtype and got.shape == want.shape
        if not want.numel():
            continue
        got = got.double().cpu()
        assert torch.isfinite(got).all(), name
        bound = (relative + (HALF_STEP if narrow else 0) + (2 * math.sqrt(count) + 8) * U) * terms + (HALF_STEP if narrow else U) * want.abs()
        worst = float(((got - want).abs() / (bound + 1e-30)).max())
        assert worst <= 1, f"{name}: {worst:.2f} times the bound"
        rms = float(want.square().mean().sqrt())
        mean = float((got - want).abs().mean()) / (rms or 1.0)
        assert mean <= (2 * HALF_STEP if narrow else relative + 8 * U * math.sqrt(count + 16)), f"{name}: mean {mean:.2e}"
    assert not g["dx"].cpu()[~live].any()


def weights(T, seed=5):
    g = generator(seed)
    return torch.rand(T, device="cuda", generator=g) + 0.5, 0.3 * torch.randn(T, device="cuda", generator=g)


# around tiles of 64, 128 and 256 tokens and rows of the table, steps of 32 and 64 of dim, sixteen bytes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 2, 3), (2, 1, 64), (3, 255, 31), (5, 256, 32), (17, 257, 33), (63, 127, 63), (64, 128, 64),
                                   (65, 129, 65), (64, 1000, 128), (66, 1000, 96), (100, 300, 100), (255, 513, 257), (256, 512, 256),
                                   (257, 700, 385), (300, 5000, 192), (1024, 600, 70), (1025, 1500, 64), (700, 3001, 513)])
def test_sizes(lb, dtype, T, V, D):
    x, w, y = inputs(T, V, D, TYPES[dtype], seed=T + V)
    dloss, dlse = weights(T)
    check(lb, x, w, y, dloss=dloss, dlse=dlse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 40, 64, 65, 300, 1500, 2100])
@pytest.mark.parametrize("ignored", [0.3, 0.95, 1.0])
def test_ignored_tokens(lb, dtype, T, ignored):
    """They are left out, whatever their rows hold."""
    x, w, y = inputs(T, 400, 72, TYPES[dtype], seed=T, ignored=ignored)
    y[::7] = 400
    dead = (y < 0) | (y >= 400)
    x[dead] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda")[torch.arange(int(dead.sum()), device="cuda") % 3][:, None].to(x.dtype)
    dloss, dlse = weights(T)
    dloss[dead], dlse[dead] = float("nan"), float("inf")
    check(lb, x, w, y, dloss=torch.where(dead, 0, dloss), dlse=torch.where(dead, 0, dlse))
    lse = lb.lbscan_loss_fwd(x, w, y)[1]
    a, b = (lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=torch.where(dead, fill, dloss), dlse=dlse) for fill in (0.0, float("nan")))
    assert torch.equal(a["dx"], b["dx"]) and torch.equal(a["dweight"], b["dweight"]) and torch.isfinite(a["dweight"]).all()


@pytest.mark.parametrize("far", [-(1 << 62), -1, 200, 1 << 31, (1 << 32) + 5, (1 << 62)])
def test_targets_of_64_bits(lb, far):
    x, w, y = inputs(70, 200, 64, torch.float32)
    y[3], y[69] = far, far
    check(lb, x, w, y, dloss=weights(70)[0])


@pytest.mark.parametrize("T,V", [(50, 300), (300, 700)])
def test_targets_of_32_bits(lb, T, V):
    x, w, y = inputs(T, V, 100, torch.bfloat16, ignored=0.2)
    a, b = lb.lbscan_loss_fwd(x, w, y), lb.lbscan_loss_fwd(x, w, y.int())
    assert all(torch.equal(*p) for p in zip(a, b))
    check(lb, x, w, y.int(), dloss=weights(T)[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.125, -1.5, 0.0])
def test_scales(lb, dtype, scale):
    x, w, y = inputs(90, 333, 64, TYPES[dtype])
    check(lb, x, w, y, scale=scale, dloss=weights(90)[0], dlse=weights(90)[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("peak", [0.0, 1e-3, 30.0])
def test_flat_and_peaked_logits(lb, dtype, peak):
    x, w, y = inputs(70, 600, 128, TYPES[dtype], peak=peak)
    check(lb, x, w, y, dloss=weights(70)[0])


def test_one_gradient_alone(lb):
    x, w, y = inputs(300, 500, 64, torch.float32)
    dloss, dlse = weights(300)
    check(lb, x, w, y, dloss=dloss)
    check(lb, x, w, y, dlse=dlse)
    check(lb, x, w, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 65])
def test_alignment_and_margins(lb, dtype, D):
    x, w, y = inputs(80, 300, D, TYPES[dtype])
    check(lb, off_by_one(x), off_by_one(w), off_by_one(y), dloss=off_by_one(weights(80)[0]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(3, 130, 33), (90, 700, 65), (300, 300, 130)])
def test_nothing_is_written_beside(lb, dtype, T, V, D):
    """Through the C entry, with margins around every output and exactly the scratch that is asked for."""
    import ctypes
    x, w, y = inputs(T, V, D, TYPES[dtype], ignored=0.2)
    dloss = weights(T)[0]
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    want = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=dloss)
    lib = lb.load()
    outs = {k: guarded(torch.full_like(v, 7)) for k, v in dict(loss=loss, lse=lse, **want).items()}
    a = lb.LbscanLossArgs()
    a.tokens, a.vocab, a.dim, a.dtype, a.ids_type, a.scale = T, V, D, int(dtype == "bf16"), 1, 1.0
    a.x, a.weight, a.targets, a.loss, a.lse = (t.data_ptr() for t in (x, w, y, outs["loss"][0], outs["lse"][0]))
    for which in (0, 1):
        room, stands = guarded(torch.zeros(lib.lbscan_loss_workspace_bytes(ctypes.byref(a), which), dtype=torch.uint8, device="cuda"), 256)
        a.workspace, a.workspace_bytes = room.data_ptr(), room.numel()
        torch.cuda.synchronize()
        if which == 0:
            assert lib.lbscan_loss_fwd(ctypes.byref(a), None) == 0
        else:
            assert lib.lbscan_loss_bwd(ctypes.byref(a), dloss.data_ptr(), None, outs["dx"][0].data_ptr(), outs["dweight"][0].data_ptr(), None) == 0
        torch.cuda.synchronize()
        assert stands()
    for k, v in dict(loss=loss, lse=lse, **want).items():
        assert outs[k][1]() and torch.equal(outs[k][0], v), k


def test_empty_sizes(lb):
    for T, V in ((0, 10), (5, 0), (0, 0)):
        x, w = torch.randn(T, 8, device="cuda"), torch.randn(V, 8, device="cuda")
        y = torch.zeros(T, dtype=torch.int64, device="cuda")
        loss, lse = lb.lbscan_loss_fwd(x, w, y)
        assert loss.shape == lse.shape == (T,) and not loss.any() and not lse.any()
        g = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=loss)
        assert g["dx"].shape == (T, 8) and g["dweight"].shape == (V, 8) and not g["dx"].any() and not g["dweight"].any()


def test_infinite_and_nan_logits(lb):
    """A token whose row holds NaN has NaN; the losses of the others stand.  A row of the table of minus infinities has no weight."""
    x, w, y = inputs(80, 300, 64, torch.float32)
    want = lb.lbscan_loss_fwd(x, w, y)
    x[7, 3] = float("nan")
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    others = torch.arange(80, device="cuda") != 7
    assert torch.isnan(loss[7]) and torch.isnan(lse[7]) and torch.equal(loss[others], want[0][others])
    x, w, y = inputs(80, 300, 64, torch.float32)
    x = x.abs() + 0.1
    y.clamp_(max=298)
    want = lb.lbscan_loss_fwd(x, w[:299].contiguous(), y)
    w[299] = -float("inf")
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    assert torch.allclose(loss, want[0], rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("dtype", TYPES)
def test_autograd(lb, dtype):
    from paper_2506_15976_amd.autograd import linear_cross_entropy
    x, w, y = inputs(90, 300, 64, TYPES[dtype], ignored=0.2)
    x3 = x.view(3, 30, 64).requires_grad_(True)
    w.requires_grad_(True)
    loss, lse = linear_cross_entropy(x3, w, y.view(3, 30), scale=0.5)
    assert loss.shape == lse.shape == (3, 30)
    n = (y >= 0).sum()
    dx, dw = torch.autograd.grad(loss.sum() / n + 1e-2 * (lse ** 2).sum() / n, (x3, w))
    d = torch.ones(90, device="cuda") / n
    want = lb.lbscan_loss_bwd(x, w, y, lse=lse.detach().view(-1), dloss=d, dlse=(2e-2 * lse.detach().view(-1)) / n, scale=0.5)
    assert torch.allclose(dx.view(90, 64).float(), want["dx"].float(), rtol=2e-2, atol=1e-6)
    assert torch.allclose(dw.float(), want["dweight"].float(), rtol=2e-2, atol=1e-6)
    # one of the two alone; tensors that are not dense; second derivatives
    only = torch.autograd.grad(linear_cross_entropy(x.detach(), w, y, scale=0.5)[0].sum(), w)[0]
    rows = torch.cat([x.detach(), x.detach()], 1)[:, :64].requires_grad_(True)
    both = torch.autograd.grad(linear_cross_entropy(rows, w, y, scale=0.5)[0].sum(), (rows, w))
    assert torch.equal(only, both[1])
    with pytest.raises(lb.LbscanError):
        torch.autograd.grad(linear_cross_entropy(x3, w, y.view(3, 30))[0].sum(), x3, create_graph=True)


def test_differences(lb):
    """The gradients against differences of the kernels' own losses, in a direction of rows and table."""
    x, w, y = inputs(40, 70, 32, torch.float32, peak=1.0)
    g = generator(8)
    dx, dw = torch.randn(40, 32, device="cuda", generator=g), torch.randn(70, 32, device="cuda", generator=g)
    lse = lb.lbscan_loss_fwd(x, w, y)[1]
    grads = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=torch.ones(40, device="cuda"))
    slope = float((grads["dx"] * dx).double().sum() + (grads["dweight"] * dw).double().sum())
    h = 2.0 ** -8
    up, down = (lb.lbscan_loss_fwd(x + s * h * dx, w + s * h * dw, y)[0].double().sum() for s in (1, -1))
    # losses of about 5 are off by 1e-6 each, 40 of them by 6e-6; over 2 h: 8e-4.  The difference's own error is h^2 / 6 of the third
    # derivative in this direction, some hundreds: 1e-3 of them
    assert abs(float(up - down) / (2 * h) - slope) <= 5e-3 * abs(slope) + 0.5


def test_errors_are_those_of_the_results_own_rounding(lb):
    """bf16, few words that many tokens have: the 2-norm of the error over that of the result.  A rounding to bf16 of values with
    mantissas by 1/m has the error 2^-7 sqrt(1/12 * 3 / (8 ln 2)) = 1.66e-3; the terms of G beside the targets', rounded once
    themselves, have less than a tenth of the energy here (sum of p^2 below 0.01): 1.67e-3, to 2^-9 = 1.95e-3."""
    x, w, _ = inputs(4000, 3000, 256, torch.bfloat16)
    y = (torch.rand(4000, device="cuda", generator=generator(4)) ** 4 * 3000).long().clamp(max=2999)
    d = weights(4000)[0]
    lse = lb.lbscan_loss_fwd(x, w, y)[1]
    got = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=d)
    G = torch.softmax(x.double() @ w.double().T, 1) * d.double()[:, None]
    G[torch.arange(4000, device="cuda"), y] -= d.double()
    for name, want in (("dx", G @ w.double()), ("dweight", G.T @ x.double())):
        assert float((got[name].double() - want).norm() / want.norm()) <= 2.0 ** -9, name


def test_same_bits_twice(lb):
    x, w, y = inputs(3000, 5000, 320, torch.bfloat16, ignored=0.1)
    d = weights(3000)[0]
    runs = []
    for _ in range(2):
        loss, lse = lb.lbscan_loss_fwd(x, w, y)
        runs.append([loss, lse, *lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=d).values()])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_the_vocabulary(lb, dtype):
    """Tokens enough that G has room for a part of the vocabulary at a time: rows of gradients as of small calls."""
    V, D = 5000, 64
    T = 1 << 17
    x, w, y = inputs(T, V, D, TYPES[dtype])
    from paper_2506_15976_amd import binding
    import ctypes
    a = binding.LbscanLossArgs(T, V, D, int(dtype == "bf16"), 1, 1.0, x.data_ptr(), w.data_ptr(), y.data_ptr(), None, None, None, 0)
    assert lb.load().lbscan_loss_workspace_bytes(ctypes.byref(a), 1) < 2 * (1 << 30)
    d = torch.rand(T, device="cuda")
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    g = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=d)
    some = torch.arange(0, T, 1999, device="cuda")
    want = [t[some] for t in (loss, lse, g["dx"])]
    few = lb.lbscan_loss_fwd(x[some].contiguous(), w, y[some])
    dx = lb.lbscan_loss_bwd(x[some].contiguous(), w, y[some], lse=few[1], dloss=d[some])["dx"]
    assert torch.allclose(few[0], want[0], rtol=1e-5, atol=1e-5) and torch.allclose(few[1], want[1], rtol=1e-5, atol=1e-5)
    step = 2 * HALF_STEP if dtype == "bf16" else 1e-5
    assert float((dx.float() - want[2].float()).abs().max()) <= 2 * step * float(dx.float().abs().max())
    # dweight: plain, a piece of the tokens at a time
    plain = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    sizes = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    for k in range(0, T, 8192):
        xs, ys, ds = x[k:k + 8192].double(), y[k:k + 8192], d[k:k + 8192].double()
        p = torch.softmax(xs @ w.double().T, 1) * ds[:, None]
        sizes += p.T @ xs.abs()
        sizes.index_add_(0, ys, xs.abs() * ds[:, None])
        p.scatter_add_(1, ys[:, None], -ds[:, None])
        plain += p.T @ xs
    bound = (1e-4 + (HALF_STEP if dtype == "bf16" else 0)) * sizes + (HALF_STEP if dtype == "bf16" else U) * plain.abs()
    assert bool(((g["dweight"].double() - plain).abs() <= bound).all())


def test_replayed_in_a_graph(lb):
    x, w, y = inputs(700, 900, 128, torch.bfloat16, ignored=0.3)
    d = weights(700)[0]

    def both():
        loss, lse = lb.lbscan_loss_fwd(x, w, y)
        return [loss, lse, *lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=d).values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        x.normal_()
        y.copy_(torch.where(torch.rand(700, device="cuda") < 0.3 * k, -1, torch.randint(0, 900, (700,), device="cuda")))
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_on_named_streams(lb):
    """Two calls at once, each on a stream of its own."""
    x, w, y = inputs(700, 900, 128, torch.float32)
    d = weights(700)[0]
    want = lb.lbscan_loss_fwd(x, w, y)
    grads = lb.lbscan_loss_bwd(x, w, y, lse=want[1], dloss=d)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [lb.lbscan_loss_fwd(x, w, y, stream=s) for s in streams]
    more = [lb.lbscan_loss_bwd(x, w, y, lse=r[1], dloss=d, stream=s) for r, s in zip(got, streams)]
    torch.cuda.synchronize()
    for r, m in zip(got, more):
        assert torch.equal(r[0], want[0]) and torch.equal(r[1], want[1])
        assert torch.equal(m["dx"], grads["dx"]) and torch.equal(m["dweight"], grads["dweight"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(5, 300, 40), (70, 600, 64), (300, 700, 96)])
def test_rows_of_the_table_that_are_minus_infinity(lb, dtype, T, V, D):
    """Words that are masked by their rows (tokens of positive elements): no probability, no gradient, loss and the other rows'
    gradients as of the table without them."""
    x, w, y = inputs(T, V, D, TYPES[dtype])
    x, gone = x.abs() + 0.01, torch.arange(0, V, 7, device="cuda")
    keep = torch.ones(V, dtype=torch.bool, device="cuda")
    keep[gone] = False
    y = torch.nonzero(keep)[:, 0][y % int(keep.sum())]
    masked = w.clone()
    masked[gone] = -math.inf
    loss, lse = lb.lbscan_loss_fwd(x, masked, y)
    d = weights(T)[0]
    g = lb.lbscan_loss_bwd(x, masked, y, lse=lse, dloss=d)["dweight"]
    assert torch.isfinite(loss).all() and torch.isfinite(g).all() and not g[gone].any()
    number = torch.cumsum(keep, 0) - 1
    check(lb, x, w[keep].contiguous(), number[y])
    other = lb.lbscan_loss_fwd(x, w[keep].contiguous(), number[y])
    # (a sum in another order: the bound of the logits, as in check)
    size = float((x.double().abs() @ w[keep].double().abs().T).max())
    limit = 2 * (2 * math.sqrt(D) + 8) * U * size + 16 * U * float(lse.abs().max())
    assert float((lse - other[1]).abs().max()) <= limit and float((loss - other[0]).abs().max()) <= 2 * limit
    want = lb.lbscan_loss_bwd(x, w[keep].contiguous(), number[y], lse=other[1], dloss=d)["dweight"]
    p = torch.softmax(x.double() @ w[keep].double().T, 1) * d[:, None]
    p[torch.arange(T, device="cuda"), number[y]] += d.double()
    terms = p.T @ x.double().abs()
    step = HALF_STEP if x.dtype == torch.bfloat16 else U
    relative = 2 * limit + 8 * U * (1 + float(lse.abs().max())) + (2 * math.sqrt(T) + 8) * U + (HALF_STEP if x.dtype == torch.bfloat16 else 0)
    assert bool(((g[keep].double() - want.double()).abs() <= 2 * relative * terms + 2 * step * want.double().abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("before", [1, 8, 64])
@pytest.mark.parametrize("T,V,D", [(1, 129, 64), (7, 300, 65), (40, 257, 33), (64, 700, 100), (64, 1100, 257), (65, 300, 100), (33, 130, 1)])
def test_tables_between_no_numbers(lb, dtype, before, T, V, D):
    """Rows of any length and address, read where they are or copied: what stands in front of and behind them is not used."""
    def between(t):
        flat = torch.full((t.numel() + before + 64,), math.nan, device="cuda", dtype=t.dtype)
        inner = flat[before:before + t.numel()].view(t.shape)
        inner.copy_(t)
        return inner
    x, w, y = inputs(T, V, D, TYPES[dtype], ignored=0.1)
    check(lb, between(x), between(w), y, dloss=weights(T)[0], dlse=weights(T)[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", [(40, 64), (40, 65), (64, 130), (1, 33)])
def test_few_tokens_replayed_in_a_graph(lb, dtype, T, D):
    x, w, y = inputs(T, 500, D, TYPES[dtype])
    d, e = weights(T)

    def both():
        loss, lse = lb.lbscan_loss_fwd(x, w, y)
        return [loss, lse, *lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=d, dlse=e).values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        x.normal_()
        y.copy_(torch.where(torch.rand(T, device="cuda") < 0.3 * k, 500, torch.randint(0, 500, (T,), device="cuda")))
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))

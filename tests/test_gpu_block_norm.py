"""The norms around a block on the GPU against the 64-bit reference: every family of launch shapes, every set of options,
gradients, absent parameters, more rows than teams, in place, any alignment, graphs, streams."""
import itertools

import pytest
import torch

import model_reference as ref
from model_util import NORM, NORM_GRADIENT, TYPES, close_terms, generator, guarded
from sequence_util import close, off_by_one, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def inputs(rows, dim, dtype, *, gate=True, residual=True, weight=True, branch_weight=True, seed=0):
    g = generator(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    t = dict(x=rand(rows, dim).to(dtype))
    if weight:
        t["weight"] = 1 + 0.3 * rand(dim)
    if gate:
        t["gate"] = rand(rows, dim).to(dtype)
    if branch_weight:
        t["branch_weight"] = 0.7 + 0.2 * rand(dim)
    if residual:
        t["residual"] = 2 * rand(rows, dim) + 0.3
    return t


NAMES = {"x": "dx", "weight": "dweight", "gate": "dgate", "branch_weight": "dbranch_weight", "residual": "dresidual"}


def check(lb, t, with_dsum=True, **options):
    x = t["x"]
    g = generator(77)
    dout = torch.randn(x.shape, device="cuda", generator=g).to(x.dtype)
    dsum = torch.randn(x.shape, device="cuda", generator=g) if "residual" in t and with_dsum else None
    want, grads = ref.gradients(lambda **k: ref.block_norm(**k, **options), t, (dout, dsum))
    _, terms = ref.gradients(lambda **k: ref.block_norm(**k, frozen=True, **options), t, (dout, dsum))
    r = lb.lbscan_block_norm_fwd(**t, return_stats=True, **options)
    total = r[1] if "residual" in t else None
    close(r[0], to_numpy(want[0]), NORM[x.dtype], "y")
    if total is not None:
        close(total, to_numpy(want[1]), NORM[torch.float32], "sum")
    options.pop("eps", None)
    d = lb.lbscan_block_norm_bwd(x, t.get("weight"), dout=dout, gate=t.get("gate"), branch_weight=t.get("branch_weight"),
                                 total=total, dsum=dsum, branch_rstd=r[-2], stream_rstd=r[-1], **options)
    for k, name in NAMES.items():
        assert (d[name] is not None) == (k in t), name
        if k in t:
            close_terms(d[name], grads[k], terms[k], NORM_GRADIENT[d[name].dtype], name)


# a team of 16 lanes with one element and with a pack; a wave; two, four, eight; beyond registers (backward, forward)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 7, 16, 33, 64, 65, 100, 200, 257, 384, 500, 768, 1000, 1024, 1025, 1500, 2050, 4000, 4096, 4100,
                                 6000, 8192, 8193, 10000, 12288, 12289])
def test_widths(lb, dtype, dim):
    check(lb, inputs(5, dim, TYPES[dtype], seed=dim), norm_branch=True, residual_scale=0.6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [10, 200, 1030, 3000, 9000, 13000])
@pytest.mark.parametrize("gate,residual,norm_branch,norm_stream", itertools.product([False, True], repeat=4))
def test_options(lb, dtype, dim, gate, residual, norm_branch, norm_stream):
    t = inputs(3, dim, TYPES[dtype], gate=gate, residual=residual, weight=norm_stream)
    check(lb, t, norm_branch=norm_branch, norm_stream=norm_stream)


@pytest.mark.parametrize("weight,branch_weight", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("dim", [96, 1600, 12500])
def test_absent_weights(lb, weight, branch_weight, dim):
    check(lb, inputs(4, dim, torch.float32, weight=weight, branch_weight=branch_weight), norm_branch=True)
    check(lb, inputs(4, dim, torch.float32, weight=weight, branch_weight=branch_weight), with_dsum=False, norm_branch=True)


@pytest.mark.parametrize("rows,dim", [(40000, 24), (9000, 130), (5000, 700), (3001, 1300), (1501, 2500), (1100, 5000), (700, 12400)])
def test_more_rows_than_teams(lb, rows, dim):
    """(and a number of rows that the teams of a block do not divide)"""
    check(lb, inputs(rows, dim, torch.bfloat16), norm_branch=True, residual_scale=1.5)


@pytest.mark.parametrize("dim", [5, 70, 300, 1027, 2051, 9001, 12301])
def test_alignment_and_margins(lb, dim):
    t = {k: off_by_one(v) for k, v in inputs(4, dim, torch.bfloat16).items()}
    check(lb, t, norm_branch=True)
    out, stands = guarded(torch.zeros(4, dim, device="cuda", dtype=torch.bfloat16))
    got = lb.lbscan_block_norm_fwd(**t, norm_branch=True, out=out)[0]
    assert stands() and torch.equal(got, lb.lbscan_block_norm_fwd(**t, norm_branch=True)[0])


def test_sum_in_place_of_the_residual(lb):
    """Through the C entry: the stream is updated where it stands, also where the last columns are held twice."""
    import ctypes
    lib = lb.load()
    for dim in (66, 1029, 2051, 4103, 9001, 12301):
        for branch in (0, 1):
            t = inputs(300, dim, torch.float32, seed=dim)
            y, total = lb.lbscan_block_norm_fwd(**t, norm_branch=bool(branch))
            mine = torch.empty_like(y)
            a = lb.LbscanBlockNormArgs()
            a.rows, a.dim, a.norm_branch, a.norm_stream, a.eps, a.residual_scale = 300, dim, branch, 1, 1e-5, 1.0
            a.x, a.gate, a.residual, a.y, a.sum = (v.data_ptr() for v in (t["x"], t["gate"], t["residual"], mine, t["residual"]))
            a.weight, a.branch_weight = t["weight"].data_ptr(), t["branch_weight"].data_ptr()
            torch.cuda.synchronize()
            assert lib.lbscan_block_norm_fwd(ctypes.byref(a), None) == 0
            torch.cuda.synchronize()
            assert torch.equal(mine, y) and torch.equal(t["residual"], total), (dim, branch)


def test_rows_of_zeros_and_large_values(lb):
    t = inputs(4, 80, torch.float32, residual=False)
    t["x"][0] = 0
    t["x"][1] *= 1e15
    t["gate"][2], t["gate"][3] = 90.0, -90.0                  # (a closed gate: its sigmoid is 0 in fp32, to 1e-39)
    check(lb, t, norm_branch=True, eps=1e-5)


def test_no_rows_and_no_columns(lb):
    for rows, dim in ((0, 40), (3, 0)):
        t = inputs(rows, dim, torch.float32)
        y, total, rv, rs = lb.lbscan_block_norm_fwd(**t, norm_branch=True, return_stats=True)
        assert y.shape == total.shape == (rows, dim) and not rv.any() and not rs.any()
        d = lb.lbscan_block_norm_bwd(t["x"], t["weight"], dout=y, gate=t["gate"], branch_weight=t["branch_weight"], total=total,
                                     branch_rstd=rv, stream_rstd=rs, norm_branch=True)
        assert not d["dweight"].any() and not d["dbranch_weight"].any() and d["dx"].shape == (rows, dim)


def test_offsets_beyond_2_31(lb):
    """More than 2^31 elements a tensor: the last rows are those of a small call."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    dim, rows = 4096, (1 << 31) // 4096 + 5
    x = torch.randn(rows, dim, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(dim, device="cuda")
    y, _, rs = lb.lbscan_block_norm_fwd(x, w, return_stats=True)
    small = lb.lbscan_block_norm_fwd(x[-9:].clone(), w, return_stats=True)
    assert torch.equal(y[-9:], small[0]) and torch.equal(rs[-9:], small[2])
    d = lb.lbscan_block_norm_bwd(x, w, dout=y, stream_rstd=rs)
    e = lb.lbscan_block_norm_bwd(x[-9:].clone(), w, dout=small[0], stream_rstd=small[2])
    assert torch.equal(d["dx"][-9:], e["dx"])
    del x, y, d
    torch.cuda.empty_cache()


@pytest.mark.parametrize("residual", [False, True])
def test_autograd(lb, residual):
    from paper_2506_15976_amd.autograd import block_norm
    t = inputs(6, 90, torch.float32, residual=residual)
    leaves = {k: v.clone().requires_grad_(True) for k, v in t.items()}
    out = block_norm(**leaves, norm_branch=True, residual_scale=0.5)
    downs = [torch.randn(6, 90, device="cuda") for _ in range(1 + residual)]
    grads = torch.autograd.grad(out, list(leaves.values()), downs)
    _, want = ref.gradients(lambda **k: ref.block_norm(**k, norm_branch=True, residual_scale=0.5), t, downs)
    for g, k in zip(grads, leaves):
        close(g, to_numpy(want[k]), NORM_GRADIENT[torch.float32], k)
    # the stream's gradient alone, and a gradient that is not dense
    if residual:
        y, s = block_norm(**leaves, norm_branch=True)
        only = torch.autograd.grad(s, list(leaves.values()), downs[1].t().contiguous().t())
        _, want = ref.gradients(lambda **k: ref.block_norm(**k, norm_branch=True), t, (torch.zeros(6, 90), downs[1]))
        for g, k in zip(only, leaves):
            close(g, to_numpy(want[k]), NORM_GRADIENT[torch.float32], k)
    x = t["x"].clone().requires_grad_(True)
    y = block_norm(x.view(2, 3, 90), t["weight"])
    with pytest.raises(lb.LbscanError):
        torch.autograd.grad(y.sum(), x, create_graph=True)


def test_same_bits_twice(lb):
    t = inputs(5000, 768, torch.bfloat16)
    runs = []
    for _ in range(2):
        y, total, rv, rs = lb.lbscan_block_norm_fwd(**t, norm_branch=True, return_stats=True)
        d = lb.lbscan_block_norm_bwd(t["x"], t["weight"], dout=y, gate=t["gate"], branch_weight=t["branch_weight"], total=total,
                                     dsum=total, branch_rstd=rv, stream_rstd=rs, norm_branch=True)
        runs.append([y, total, *d.values()])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_replayed_in_a_graph(lb):
    t = inputs(300, 768, torch.bfloat16)

    def both():
        y, total, rv, rs = lb.lbscan_block_norm_fwd(**t, norm_branch=True, return_stats=True)
        d = lb.lbscan_block_norm_bwd(t["x"], t["weight"], dout=y, gate=t["gate"], branch_weight=t["branch_weight"], total=total,
                                     branch_rstd=rv, stream_rstd=rs, norm_branch=True)
        return [y, total, *d.values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(4):
        t["x"].normal_()
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_on_a_named_stream(lb):
    t = inputs(300, 768, torch.float32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    y, total, rv, rs = lb.lbscan_block_norm_fwd(**t, norm_branch=True, return_stats=True, stream=side)
    d = lb.lbscan_block_norm_bwd(t["x"], t["weight"], dout=y, gate=t["gate"], branch_weight=t["branch_weight"], total=total,
                                 branch_rstd=rv, stream_rstd=rs, norm_branch=True, stream=side)
    side.synchronize()
    want = lb.lbscan_block_norm_fwd(**t, norm_branch=True)
    assert torch.equal(y, want[0]) and torch.equal(total, want[1]) and torch.isfinite(d["dx"]).all()

"""Layer norm of more rows of more columns than registers hold than one launch has threads for (32 bits of them along an
axis of its grid)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    yield pkg
    torch.cuda.empty_cache()          # (the blocks are large)


def test_many_long_rows(lb):
    rows, dim, period = (1 << 22) + 5, 12289, 37
    if torch.cuda.mem_get_info()[0] < 230e9:
        pytest.skip("needs 230 GB of device memory")
    one = torch.randn(period, dim, device="cuda").bfloat16()
    x = torch.empty(rows, dim, device="cuda", dtype=torch.bfloat16)
    whole = rows // period * period
    x[:whole].view(-1, period, dim).copy_(one.expand(whole // period, -1, -1))
    x[whole:].copy_(one[:rows - whole])
    want, mean, rstd = lb.lbscan_norm_fwd(one, return_stats=True)

    def check(v, w, what):
        assert torch.equal(v[whole:], w[:rows - whole]), what
        assert all(bool((p == w).all()) for p in v[:whole].view(-1, *w.shape).split(1024)), what

    y, means, rstds = lb.lbscan_norm_fwd(x, return_stats=True, out=x)
    check(y, want, "y")
    check(means, mean, "mean")
    check(rstds, rstd, "rstd")
    # the gradient of y = x: any rows will do, these are in memory
    g = lb.lbscan_norm_bwd(y, dout=y, mean=means, rstd=rstds, with_bias=False)
    check(g["dx"], lb.lbscan_norm_bwd(want, dout=want, mean=mean, rstd=rstd, with_bias=False)["dx"], "dx")

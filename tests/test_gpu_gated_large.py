"""The gated recurrence over more rows than one launch has threads for (32 bits of them along an axis of its grid)."""
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


def test_many_rows(lb):
    """Eight lanes a row, and rows that differ from one another as far as the middle of them; about 50 GB."""
    rows, L, period = (1 << 29) + 40, 8, 100003
    if torch.cuda.mem_get_info()[0] < 80e9:
        pytest.skip("needs 80 GB of device memory")
    one = torch.randn(period, L, device="cuda").bfloat16()
    decay_of_one = torch.linspace(-6.0, 1.0, period, device="cuda")
    x = torch.empty(1, rows, L, device="cuda", dtype=torch.bfloat16)
    decay = torch.empty(rows, device="cuda")
    whole = rows // period * period
    x[0, :whole].view(-1, period, L).copy_(one.expand(whole // period, -1, -1))
    x[0, whole:].copy_(one[:rows - whole])
    decay[:whole].view(-1, period).copy_(decay_of_one.expand(whole // period, -1))
    decay[whole:].copy_(decay_of_one[:rows - whole])
    y = lb.lbscan_gated_fwd(x, x, x, decay)
    g = lb.lbscan_gated_bwd(x, x, x, decay, dout=y)
    # calls of fewer rows; whole blocks of 32 rows, as rows that share a wave share the way their gates are computed
    for part in range(0, rows, 1 << 25):
        some = slice(part, part + (1 << 25))
        u, d = x[:, some], decay[some]
        assert torch.equal(lb.lbscan_gated_fwd(u, u, u, d), y[:, some]), part
        for k, want in lb.lbscan_gated_bwd(u, u, u, d, dout=y[:, some]).items():
            assert torch.equal(want, g[k][some] if k == "ddecay" else g[k][:, some]), (k, part)

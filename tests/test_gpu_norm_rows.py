"""Layer norm of more rows than the grid has teams, for every team: each walks several rows with the next ones' loads
under way."""
import pytest
import torch

import sequence_reference as ref
from sequence_util import NORM, TYPES, close, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


# the forward grid has 2048 blocks: of sixteen teams of 16 lanes, of four waves, and of one row where a team has more waves
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,dim", [(33001, 5), (33001, 64), (8250, 200), (8250, 1000), (2101, 1500), (2101, 2100), (2101, 4000),
                                      (2101, 4200), (2101, 8200)])
def test_rows(lb, rows, dim, residual, dtype):
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(rows, dim, generator=g).to(TYPES[dtype]).cuda()
    w, b = (1 + 0.3 * torch.randn(dim, generator=g)).cuda(), torch.randn(dim, generator=g).cuda()
    r = (2 * torch.randn(rows, dim, generator=g) + 0.5).cuda() if residual else None
    dout = torch.randn(rows, dim, generator=g).to(TYPES[dtype]).cuda()
    dsum = torch.randn(rows, dim, generator=g).cuda() if residual else None
    res = lb.lbscan_norm_fwd(x, w, b, residual=r, return_stats=True)
    total = res[1] if residual else None
    got = lb.lbscan_norm_bwd(None if residual else x, w, dout=dout, mean=res[-2], rstd=res[-1], total=total, dsum=dsum)
    # all columns' sums, and the rows that a team takes first, second and last
    s = to_numpy(x if total is None else total)
    want = ref.norm_bwd(s, to_numpy(w), to_numpy(dout), None if dsum is None else to_numpy(dsum))
    close(got["dweight"], want["dweight"], NORM["fp32"], "dweight")
    close(got["dbias"], want["dbias"], NORM["fp32"], "dbias")
    for part in (slice(0, 200), slice(2000, 2100), slice(rows - 200, rows)):
        y, sums, _, rstd = ref.norm_fwd(to_numpy(x[part]), to_numpy(w), to_numpy(b), None if r is None else to_numpy(r[part]))
        close(res[0][part], y, NORM[dtype], "y")
        close(res[-1][part], rstd, NORM["fp32"], "rstd")
        close(got["dx"][part], want["ds"][part], NORM[dtype], "dx")
        if residual:
            close(total[part], sums, NORM["fp32"], "sum")
            close(got["dresidual"][part], want["ds"][part], NORM["fp32"], "dresidual")

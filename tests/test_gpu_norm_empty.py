"""Statistics of rows without columns are zeros, not what the memory held."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("side", [False, True])
@pytest.mark.parametrize("residual", [False, True])
def test_no_columns(residual, side):
    import paper_2506_15976_amd as lb
    s = torch.cuda.Stream() if side else None
    x = torch.empty(4000, 0, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        dirty = [torch.full((4000,), 7.0, device="cuda") for _ in range(8)]
    del dirty
    res = lb.lbscan_norm_fwd(x, residual=x if residual else None, return_stats=True, stream=s)
    torch.cuda.synchronize()
    assert res[0].shape == (4000, 0) and res[-1].shape == res[-2].shape == (4000,)
    assert not res[-1].any() and not res[-2].any()
    g = lb.lbscan_norm_bwd(None if residual else x, dout=x, mean=res[-2], rstd=res[-1], total=x if residual else None)
    assert g["dx"].shape == (4000, 0)

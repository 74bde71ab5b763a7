"""Scans of more rows than one launch has threads for (32 bits of them along an axis of its grid) raise an error."""
import pytest
import torch

from paper_2506_15976_amd.binding import EHIP, LbscanError

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    yield pkg
    torch.cuda.empty_cache()


@pytest.mark.parametrize("which", ["fwd", "bwd", "bidir"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_too_many_rows(lb, dtype, which):
    # a block of 256 threads has rows of one batch entry
    batch = (1 << 24) + 64
    row = torch.rand(batch, 1, 2, device="cuda").to(dtype)
    s = dict(x=row, delta=row, A=-torch.ones(1, 1, device="cuda"), Bm=row, Cm=row)
    with pytest.raises(LbscanError) as e:
        if which == "fwd":
            lb.lbscan_fwd(**s, window=4)
        elif which == "bwd":
            lb.lbscan_bwd(**s, dout=row, window=4)
        else:
            lb.lbscan_bidir_fwd(s, s)
    assert e.value.code == EHIP
    # and the next call runs
    few = {k: v if k == "A" else v[:5].contiguous() for k, v in s.items()}
    assert torch.isfinite(lb.lbscan_fwd(**few, window=4)).all()

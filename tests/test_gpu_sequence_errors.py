"""An error of a backward pass is the operators' own, with its code, also where the autograd engine's threads raise it."""
import pytest
import torch

from paper_2506_15976_amd.binding import EUNSUPPORTED, LbscanError

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("threads", [True, False])
@pytest.mark.parametrize("which", ["gated", "norm", "sum", "embed"])
def test_second_derivatives(which, threads):
    from paper_2506_15976_amd.autograd import gated_linear_recurrence, layer_norm, token_embedding
    x = torch.randn(2, 3, 40, device="cuda", requires_grad=True)
    table = torch.randn(5, 8, device="cuda", requires_grad=True)
    y, leaf = {"gated": lambda: (gated_linear_recurrence(x, x, x, torch.zeros(3, device="cuda")), x),
               "norm": lambda: (layer_norm(x), x),
               "sum": lambda: (layer_norm(x, residual=torch.zeros(2, 3, 40, device="cuda"))[1], x),
               "embed": lambda: (token_embedding(torch.zeros(7, dtype=torch.int64, device="cuda"), table), table)}[which]()
    with torch.autograd.set_multithreading_enabled(threads):
        with pytest.raises(LbscanError, match="once") as e:
            torch.autograd.grad(y.square().sum(), leaf, create_graph=True, retain_graph=True)
        assert e.value.code == EUNSUPPORTED
        # nothing is left behind
        g, = torch.autograd.grad(y.square().sum(), leaf)
    assert torch.isfinite(g).all()

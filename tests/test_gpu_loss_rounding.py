"""What rounding leaves in the gradients of the loss in bf16, in the 2-norm, against 64 bits.

A value is rounded to bf16 with an error that is as good as uniform in half a step on both sides, ulp^2 / 12 in its square.  The gradients'
error is, besides that of fp32 sums, their own rounding and that of G beside the targets, which goes into dx with the squares of the
table's rows and into dweight with those of the tokens' rows; what rounding G at the targets leaves is added by itself.  The sum of many
such squares (e^2 of a uniform e has the deviation 0.9 of its mean; an error vector of one token or row of the table, whose terms share
their factors, 1.5) is within six deviations of its mean.  The remainder at the targets, had it been dropped or added to
another row, is known from the 64-bit G: the bound tells it from noise, which is checked, too.
"""
import math

import pytest
import torch

from loss_branches import CALLS, live
from model_util import generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def step_squared(v):
    """ulp^2 / 12 of values rounded to bf16, eight bits."""
    return torch.where(v == 0, 0, torch.ldexp(torch.ones_like(v), 2 * (torch.frexp(v)[1] - 8))) / 12


class Energy:
    """A sum of squares, and the square of its deviation."""
    def __init__(self):
        self.sum, self.square = 0.0, 0.0

    def add(self, parts, deviation):
        self.sum += float(parts.sum())
        self.square += deviation ** 2 * float(parts.square().sum())
        return self

    def bound(self):
        return self.sum + 6 * math.sqrt(self.square)


def rounding(lb, x, w, y, down, *, discriminates):
    T, D = x.shape
    V = w.shape[0]
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    got = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=down)
    W, rows = w.double(), torch.nonzero((y >= 0) & (y < V))[:, 0]
    lengths = W.square().sum(1)
    dx, dw = torch.zeros(T, D, device="cuda", dtype=torch.float64), torch.zeros(V, D, device="cuda", dtype=torch.float64)
    left, by_row = torch.zeros_like(dx), torch.zeros_like(dw)               # what is left at the targets, in dx and dweight
    beside_x, beside_w = torch.zeros(T, device="cuda", dtype=torch.float64), torch.zeros(V, device="cuda", dtype=torch.float64)
    for part in rows.split(max(64, (1 << 27) // V)):
        X, ys, k = x[part].double(), y[part], torch.arange(len(part), device="cuda")
        G = torch.softmax(X @ W.T, 1) * down[part, None].double()
        G[k, ys] -= down[part].double()
        dx[part] = G @ W
        dw.addmm_(G.T, X)
        hot = G[k, ys]
        e = hot - hot.to(torch.bfloat16).double()
        left[part] = e[:, None] * W[ys]
        by_row.index_add_(0, ys, e[:, None] * X)
        s = step_squared(G)
        s[k, ys] = 0
        beside_x[part] = s @ lengths
        beside_w += s.T @ X.square().sum(1)
    for name, want, beside, lost in (("dx", dx, beside_x, left), ("dweight", dw, beside_w, by_row)):
        bound = Energy().add(step_squared(want), 0.9).add(beside, 1.5).bound()
        error = float((got[name].double() - want).square().sum())
        assert error <= bound, f"{name}: {math.sqrt(error / bound):.3f} times the bound"
        if discriminates:
            # (the dropped remainder is independent of the rest: their squares add, and twice the root of the product at six deviations
            # over as many elements as there are is small beside them)
            added, own = float(lost.square().sum()), float(step_squared(want).sum())
            assert own + added - 12 * math.sqrt(added * own / lost.count_nonzero()) > bound, f"{name}: the bound does not tell"


def call(T, V, D, ignored, *, peak, seed):
    g = generator(seed)
    x = torch.randn(T, D, device="cuda", generator=g).bfloat16()
    w = (torch.randn(V, D, device="cuda", generator=g) * (peak / math.sqrt(D))).bfloat16()
    # some rows of the table are the target of many tokens
    targets = (torch.rand(T, device="cuda", generator=g) ** 4 * V).long().clamp(max=V - 1)
    y = torch.full((T,), -1, device="cuda")
    at = torch.tensor(live(T, ignored), device="cuda")
    y[at] = targets[at]
    return x, w, y, torch.rand(T, device="cuda", generator=g) + 0.5


@pytest.mark.parametrize("T,V,D,ignored,before,last,rows", CALLS)
def test_what_rounding_the_targets_leaves_is_added(lb, T, V, D, ignored, before, last, rows):
    rounding(lb, *call(T, V, D, ignored, peak=1.0, seed=T + V), discriminates=True)


@pytest.mark.parametrize("peak", [2.0, 4.0, 6.0, 12.0])
@pytest.mark.parametrize("T,V,D", [(2000, 3000, 256), (64, 3000, 256), (60, 3000, 258)])
def test_rounding_of_peaked_rows(lb, peak, T, V, D):
    """Logits of a larger deviation: beside the target a token has other large slopes, whose rounding stays."""
    rounding(lb, *call(T, V, D, 0.0, peak=peak, seed=int(peak)), discriminates=False)

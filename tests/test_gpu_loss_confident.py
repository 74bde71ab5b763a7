"""Losses of tokens whose target has nearly all of the probability, against 64 bits.

Logits are exact here: a token is a number of few bits at one place of its row, the table has numbers of few bits there.  With
u = 2^-24: an exponent (to base 2) is a product with a factor that is off by 2 u and a difference that is rounded once, so a term of the
sum, relative to the target's, is off by 3 u of its distance from it, 8 at the most where it has weight: 24 u.  Exponentials 2 u, their
sum in four chains and the joins of its parts 10 u, the quotient, the logarithm and the factor ln2 4 u, to 48 u; a target
that is not the largest adds 3 u of its distance and the roundings of the result, to 8 u of the loss.  A certain token's loss
is zero or more, and zero where there is no other row.
"""
import pytest
import torch

from model_util import TYPES, generator

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


# few tokens with rows in place and loose, more tokens; vocabularies in whole tiles and not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 0.7, -0.9])
@pytest.mark.parametrize("T,V,D", [(40, 512, 64), (40, 512, 65), (64, 300, 64), (64, 300, 65), (7, 5, 33), (300, 1024, 64), (300, 700, 70),
                                   (1100, 40, 130)])
def test_losses_of_certain_tokens(lb, dtype, scale, T, V, D):
    g = generator(T + V + D)
    x = torch.zeros(T, D, device="cuda")
    x[:, 0] = (0.75 + torch.randint(0, 17, (T,), device="cuda", generator=g) / 64) * (1 if scale > 0 else -1)
    w = torch.randn(V, D, device="cuda", generator=g)
    rows = torch.randperm(V, device="cuda", generator=g)[:4]
    w[:, 0] = torch.randint(0, 21, (V,), device="cuda", generator=g).float()
    w[rows, 0] = torch.tensor([120.0, 119.5, 116.0, 112.0], device="cuda")
    y = rows[torch.randint(0, 8, (T,), device="cuda", generator=g).clamp(max=3) % 4].clone()
    y[: T // 2] = rows[0]
    x, w = x.to(TYPES[dtype]), w.to(TYPES[dtype])
    loss, lse = lb.lbscan_loss_fwd(x, w, y, scale=scale)
    logits = float(torch.tensor(scale)) * x[:, :1].double() @ w[:, :1].double().T
    want = torch.logsumexp(logits - logits.gather(1, y[:, None]), 1)
    assert bool((loss >= 0).all())
    worst = float(((loss.double() - want).abs() / (48 * U + 8 * U * want)).max())
    assert worst <= 1, f"{worst:.2f} times the bound"
    # lse as ever: rounded where it is added to the maximum, 8 u of itself
    exact = torch.logsumexp(logits, 1)
    assert bool(((lse.double() - exact).abs() <= 8 * U * exact.abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("D", [64, 65, 384])
@pytest.mark.parametrize("size", [1.0, 30.0])
def test_a_vocabulary_of_one(lb, dtype, T, D, size):
    """The only row there is has all of the probability: the loss is zero, lse the logit."""
    g = generator(D)
    x = (size * torch.randn(T, D, device="cuda", generator=g)).to(TYPES[dtype])
    w = torch.randn(1, D, device="cuda", generator=g).to(TYPES[dtype])
    loss, lse = lb.lbscan_loss_fwd(x, w, torch.zeros(T, device="cuda", dtype=torch.int64), scale=0.3)
    assert not loss.any() and lse.abs().max() > 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", [(50, 128), (50, 129), (700, 128)])
def test_losses_are_not_negative(lb, dtype, T, D):
    """Logits as they come, up to a few hundreds; each token's target is its largest."""
    g = generator(T + D)
    x, w = torch.randn(T, D, device="cuda", generator=g).to(TYPES[dtype]), (4 * torch.randn(900, D, device="cuda", generator=g)).to(TYPES[dtype])
    logits = x.double() @ w.double().T
    y = logits.argmax(1)
    loss, _ = lb.lbscan_loss_fwd(x, w, y)
    assert bool((loss >= 0).all()) and float(loss.min()) < 1e-3

"""Backward passes recorded into a graph that ask for some of an operator's leaves while the others are in use in an eager graph on
the default stream: they are no part of the pass, which runs."""
import pytest
import torch

from model_util import generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def operators():
    """name -> (leaves, call, the leaf that is not asked for)"""
    from paper_2506_15976_amd import autograd

    def leaf(*shape, seed):
        return torch.randn(*shape, device="cuda", generator=generator(seed)).requires_grad_(True)
    rows, table, w, gate, stream = leaf(40, 64, seed=1), leaf(90, 64, seed=2), leaf(64, seed=3), leaf(40, 64, seed=4), leaf(40, 64, seed=5)
    y = torch.randint(0, 90, (40,), device="cuda", generator=generator(6))
    x, a, b, decay = leaf(2, 16, 50, seed=7), leaf(2, 16, 50, seed=8), leaf(2, 16, 50, seed=9), leaf(16, seed=10)
    return {
        "loss, of the rows": ([rows, table], lambda: autograd.linear_cross_entropy(rows, table, y)[0], 1),
        "loss, of the table": ([rows, table], lambda: autograd.linear_cross_entropy(rows, table, y)[0], 0),
        "norms, of the rows": ([rows, w, gate, stream], lambda: autograd.block_norm(rows, w, gate=gate, residual=stream)[0], 1),
        "norms, without the stream": ([rows, w, gate, stream], lambda: autograd.block_norm(rows, w, gate=gate, residual=stream)[0], 3),
        "layer norm": ([rows, w], lambda: autograd.layer_norm(rows, w), 1),
        "gated recurrence": ([x, a, b, decay], lambda: autograd.gated_linear_recurrence(x, a, b, decay), 3),
    }


NAMES = ["loss, of the rows", "loss, of the table", "norms, of the rows", "norms, without the stream", "layer norm", "gated recurrence"]


@pytest.mark.parametrize("name", NAMES)
def test_leaves_that_the_pass_does_not_reach(lb, name):
    leaves, call, other = operators()[name]
    asked = [t for k, t in enumerate(leaves) if k != other]
    out = call()
    down = torch.randn(out.shape, device="cuda", generator=generator(11))
    want = [t.clone() for t in torch.autograd.grad(out, asked, down)]
    del out
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(call(), asked, down)
    torch.cuda.current_stream().wait_stream(side)
    alive = leaves[other] * 2.0                               # on the default stream
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(call(), asked, down)
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert alive.grad_fn is not None


@pytest.mark.parametrize("name", NAMES)
def test_leaves_that_it_reaches(lb, name):
    """The same leaf in use elsewhere and asked for: refused, whatever else is asked for."""
    leaves, call, other = operators()[name]
    down = torch.randn(call().shape, device="cuda", generator=generator(11))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(call(), leaves, down)
    torch.cuda.current_stream().wait_stream(side)
    alive = leaves[other] * 2.0
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(lb.LbscanError, match="captured"):
        with torch.cuda.graph(graph):
            torch.autograd.grad(call(), [leaves[other]], down)
    assert alive.grad_fn is not None

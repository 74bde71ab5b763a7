"""The operators of the state-space language model as it uses them together: the loss and every parameter's gradient against a plain
model in 64 bits, and prompts of different lengths and captured steps in a pool of states against whole sequences."""
import importlib.util
import math
import os

import pytest
import torch
import torch.nn.functional as F

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("state_space_lm", os.path.join(ROOT, "examples", "state_space_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def root_mean_square(x, weight):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * weight


def plain_loss(model, p, ids, targets, square):
    """The model's loss from parameters in 64 bits, a token at a time."""
    B, L = ids.shape
    table = p["table"]
    x, stream = table[ids], 0
    for k in range(model.layers):
        stream = stream + x
        x, z = (root_mean_square(stream, p[f"norm{k}"]) @ p[f"in{k}"].T).split(model.inner, -1)
        padded = F.pad(x, (0, 0, 3, 0))
        u = F.silu(sum(padded[:, j:j + L] * p[f"conv{k}"][:, j] for j in range(4)) + p[f"conv_bias{k}"])
        low, Bm, Cm = (u @ p[f"x{k}"].T).split([model.rank, model.states, model.states], -1)
        delta = F.softplus(low @ p[f"dt{k}"].T + p[f"dt_bias{k}"])
        h, rows = torch.zeros(B, model.inner, model.states, dtype=torch.float64), []
        for t in range(L):
            d = delta[:, t, :, None]
            h = torch.exp(-d * torch.exp(p[f"A{k}"])) * h + d * Bm[:, t, None] * u[:, t, :, None]
            rows.append((h * Cm[:, t, None]).sum(-1))
        y = torch.stack(rows, 1) + p[f"skip{k}"] * u
        x = root_mean_square(y * F.silu(z), p[f"gated{k}"]) @ p[f"out{k}"].T
    logits = root_mean_square(stream + x, p["norm"]) @ table.T
    there = targets >= 0
    lse = torch.logsumexp(logits, -1)
    loss = lse - logits.gather(-1, targets.clamp(min=0)[..., None])[..., 0]
    return ((loss + square * lse * lse) * there).sum() / there.sum()


# An operator's results are within about 1e-5 of their size (fp32: sums of some tens to hundreds of terms, 2^-24 each), and so are the
# products between them; 2 blocks of 9 operators and products each way, 36 in a row, add to 4e-4 where each hands on its
# input's relative error as it is.  Norms and gates do; 1e-3 leaves a factor of 2.5.
CHAIN = 1e-3


def test_gradients_of_the_model(example):
    model = example.StateSpaceLM(37, 48, 2, states=8)
    ids, targets = example.documents(5, 30, 37, torch.Generator().manual_seed(3))
    loss = model.loss(ids.cuda(), targets.cuda(), square=0.01)
    loss.backward()
    p = {k: v.detach().double().cpu().requires_grad_(True) for k, v in model.parameters.items()}
    want = plain_loss(model, p, ids, targets, 0.01)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= CHAIN * float(want.detach())
    for k, v in model.parameters.items():
        size = float(p[k].grad.abs().max())
        assert size > 0, k
        error = float((v.grad.double().cpu() - p[k].grad).abs().max())
        assert error <= CHAIN * size, (k, error / size)


def test_it_trains_in_bf16(example):
    """It runs: every step's loss and gradients are numbers, and the parameters move."""
    model = example.StateSpaceLM(32, 64, 2, dtype=torch.bfloat16)
    before = {k: v.detach().clone() for k, v in model.parameters.items()}
    losses = example.train(model, 5, vocab=32, rows=8, length=100)
    assert all(math.isfinite(v) for v in losses)
    for k, v in model.parameters.items():
        assert bool(torch.isfinite(v.grad).all()) and not torch.equal(v.detach(), before[k]), k


def test_a_pool_says_what_whole_sequences_say(example):
    """Prompts of different lengths enter free slots while others run; captured steps continue changing sets of them, in changing
    orders, with padding; a slot that is free again serves another prompt."""
    model = example.StateSpaceLM(40, 48, 2)
    server = example.Server(model, slots=7, batch=6)
    g = torch.Generator().manual_seed(11)
    ids = torch.randint(0, 40, (8, 40), generator=g).cuda()
    with torch.no_grad():
        whole = torch.stack([model.logits(model.hidden(r[None]))[0] for r in ids])
    limit = CHAIN * float(whole.std()) * 4                        # (logits of a few deviations)

    def same(logits, rows, at):
        for l, r, t in zip(logits, rows, at):
            assert float((l - whole[r, t]).abs().max()) <= limit, (r, t)

    slot, done = {}, {}

    def enter(rows, lengths, slots):
        longest = max(lengths)
        logits = server.prompt(ids[rows, :longest], torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                               torch.tensor(slots, dtype=torch.int32, device="cuda"))
        same(logits, rows, [n - 1 for n in lengths])
        slot.update(zip(rows, slots))
        done.update(zip(rows, lengths))

    def go_on(rows):
        tokens = torch.stack([ids[r, done[r]] for r in rows])
        logits = server.step(tokens, torch.tensor([slot[r] for r in rows], dtype=torch.int32, device="cuda"))
        same(logits, rows, [done[r] for r in rows])
        for r in rows:
            done[r] += 1

    enter([0, 1, 2], [1, 9, 17], [4, 0, 6])
    for _ in range(3):
        go_on([0, 1, 2])
    go_on([2, 0])
    enter([3, 4], [2, 23], [1, 2])
    for rows in ([4, 3, 2, 1, 0], [1, 3], [0], [3, 2, 4]):
        go_on(rows)
    enter([5, 6, 7], [5, 3, 8], [0, 3, 5])                        # (slot 0 was row 1's)
    for rows in ([0, 2, 3, 4, 5, 6], [7, 6, 5, 4, 3, 2], [7], [0, 5]):
        go_on(rows)


# Gradients that the convolution and the scan add up with one fp32 atomic a wave or block, in any order: of 150 tokens' terms at
# most 20 such sums a value, each rounded by 2^-24 of the terms' sizes S at most, so two runs differ by at most 40 * 2^-24 S.  150
# terms of either sign add to about S / 12; the largest of a tensor's sums is at least a third of that: 36 * 40 * 2^-24 = 9e-5.
ANY_ORDER = ("conv", "conv_bias", "A", "skip", "dt_bias")


def test_captured_training_steps(example):
    """Loss and gradients of the model from a graph, replayed with other documents between eager work: as eager steps."""
    model = example.StateSpaceLM(37, 48, 2, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    ids, targets = (t.cuda() for t in example.documents(5, 30, 37, g))
    leaves = list(model.parameters.values())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(model.loss(ids, targets), leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = model.loss(ids, targets)
        grads = torch.autograd.grad(loss, leaves)
    loss = loss.detach()
    for _ in range(4):
        for t, new in zip((ids, targets), example.documents(5, 30, 37, g)):
            t.copy_(new)
        graph.replay()
        want = model.loss(ids, targets)
        others = torch.autograd.grad(want, leaves)
        torch.cuda.synchronize()
        assert torch.equal(loss, want.detach())
        for a, b, k in zip(grads, others, model.parameters):
            if k.rstrip("01") in ANY_ORDER:
                assert float((a - b).abs().max()) <= 1e-4 * float(b.abs().max()), k
            else:
                assert torch.equal(a, b), k

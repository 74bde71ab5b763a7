"""The operators of state space language models at the ends of what they take: offsets past 32 bits, the longest row of a prompt, named
streams and their memory, outputs that share memory with inputs, recorded backward passes."""
import math
import types

import pytest
import torch

import model_reference as ref
from model_util import CONV, HALF_STEP, generator
from sequence_util import close, to_numpy

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def needs(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GB of device memory")


# ---- the loss, beyond 2^31 elements --------------------------------------------------------------------------
# x; the table; G, which has one tile of the vocabulary at the least; x and G in four bytes
@pytest.mark.parametrize("T,V,D,dtype,memory", [
    (600001, 130, 4000, torch.bfloat16, 60), (70, 700001, 4000, torch.bfloat16, 60), (5000, 560001, 4000, torch.bfloat16, 60),
    ((1 << 24) - 37, 300, 32, torch.bfloat16, 60), ((1 << 24) - 37, 140, 33, torch.float32, 100), (300, 540001, 4001, torch.float32, 100),
])
def test_loss_beyond_2_31_elements(lb, T, V, D, dtype, memory):
    """Against 64 bits, some tokens at a time; bounds as derived in test_gpu_loss.py, with dx's terms' sizes as at most
    (|g| + |g + e|) max |W|."""
    needs(memory)
    g = generator(T + V)
    x = torch.empty(T, D, device="cuda", dtype=dtype)
    for k in range(0, T, 1 << 18):
        x[k:k + (1 << 18)] = torch.randn(min(1 << 18, T - k), D, device="cuda", generator=g)
    w = torch.empty(V, D, device="cuda", dtype=dtype)
    for k in range(0, V, 1 << 18):
        w[k:k + (1 << 18)] = torch.randn(min(1 << 18, V - k), D, device="cuda", generator=g) * (2 / math.sqrt(D))
    y = torch.randint(0, V, (T,), device="cuda", generator=g)
    y[0], y[T - 1] = V - 1, 0
    down = torch.rand(T, device="cuda", generator=g) + 0.5
    loss, lse = lb.lbscan_loss_fwd(x, w, y)
    grads = lb.lbscan_loss_bwd(x, w, y, lse=lse, dloss=down)
    narrow = HALF_STEP if dtype == torch.bfloat16 else 0.0
    own = HALF_STEP if dtype == torch.bfloat16 else U
    top = float(lse.abs().max())
    tokens = [0, 1, T // 3, T - 2, T - 1] if V > 1000 else range(0, T, max(T // 500, 1))
    some = torch.tensor(sorted({*tokens, T - 1}), device="cuda")
    X, Y = x[some].double(), y[some]
    logits, size, highest = torch.empty(len(some), V, device="cuda", dtype=torch.float64), 0.0, 0.0
    for k in range(0, V, 1 << 16):
        W = w[k:k + (1 << 16)].double()
        logits[:, k:k + (1 << 16)] = X @ W.T
        size, highest = max(size, float((X.abs() @ W.abs().T).max())), max(highest, float(W.abs().max()))
    d = (2 * math.sqrt(D) + 8) * U * size
    want = torch.logsumexp(logits, 1)
    assert float((lse[some].double() - want).abs().max()) <= d + 8 * U * top
    want_loss = want - logits.gather(1, Y[:, None])[:, 0]
    assert float((loss[some].double() - want_loss).abs().max()) <= 2 * (d + 8 * U * top)
    relative = 2 * d + 8 * U * (1 + top)
    p = torch.softmax(logits, 1) * down[some, None]
    p.scatter_add_(1, Y[:, None], -down[some, None].double())
    dx = sum(p[:, k:k + (1 << 16)] @ w[k:k + (1 << 16)].double() for k in range(0, V, 1 << 16))
    terms = 2 * down[some, None].double() * highest
    bound = (relative + narrow + (2 * math.sqrt(V) + 8) * U) * terms + own * dx.abs()
    assert bool(((grads["dx"][some].double() - dx).abs() <= bound).all())
    # dweight: some rows of the table, over all tokens; the softmax's sums are those of the forward call, d off at most
    rows = torch.unique(torch.cat([torch.arange(0, V, max(V // 200, 1), device="cuda"), torch.tensor([V - 2, V - 1], device="cuda")]))
    W, plain, sizes = w[rows].double(), 0.0, 0.0
    step = (1 << 16) if D > 1000 else (1 << 20)
    for k in range(0, T, step):
        X, ys, ds = x[k:k + step].double(), y[k:k + step], down[k:k + step, None].double()
        p = torch.exp(X @ W.T - lse[k:k + step, None].double()) * ds
        hot = (ys[:, None] == rows) * ds
        plain, sizes = plain + (p - hot).T @ X, sizes + (p + hot).T @ X.abs()
    got = grads["dweight"][rows].double()
    bound = (relative + d + narrow + (2 * math.sqrt(T) + 8) * U) * sizes + own * plain.abs()
    assert bool(((got - plain).abs() <= bound).all())
    del x, w, grads, X, W, p, logits
    torch.cuda.empty_cache()


def test_longest_prompt(lb):
    """A row of as many tokens as it may have (one more is refused on the host)."""
    needs(30)
    L = (1 << 31) - 4096
    x = torch.zeros(1, 1, L, device="cuda", dtype=torch.bfloat16)
    x[..., -40:] = torch.randn(40, device="cuda", generator=generator(1))
    x[..., :9] = 1.0
    w, b = torch.randn(1, 4, device="cuda", generator=generator(2)), torch.ones(1, device="cuda")
    state = torch.ones(1, 1, 3, device="cuda", dtype=torch.bfloat16)
    y = lb.lbscan_conv1d_prompt(x, state, w, b)
    part = x[..., -30:].contiguous()
    want, after = ref.conv_prompt(part, x[..., -33:-30], w, b)
    close(y[..., -30:].contiguous(), to_numpy(want), CONV[torch.bfloat16], "the end")
    assert torch.equal(state.double().cpu(), after)
    assert len(torch.unique(y[0, 0, 12:-40][:: 1 << 12])) == 1 and len(torch.unique(y[0, 0, 0:9])) == 1
    del x, y
    torch.cuda.empty_cache()


# ---- streams ---------------------------------------------------------------------------------------------------
def calls(lb):
    """name -> a call that takes the stream and returns every tensor it made."""
    g = generator(1)

    def rand(*shape, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g).to(dtype)

    def values(r):
        return [v for v in (r.values() if isinstance(r, dict) else r) if v is not None]
    x, table, ids = rand(3000, 300), 0.1 * rand(5000, 300), torch.randint(-50, 5000, (3000,), device="cuda", generator=g)
    narrow, narrow_table = x.bfloat16(), table.bfloat16()
    lse, narrow_lse = lb.lbscan_loss_fwd(x, table, ids)[1], lb.lbscan_loss_fwd(narrow, narrow_table, ids)[1]
    down = rand(3000)
    rows, gate, stream, w = rand(3000, 640), rand(3000, 640), rand(3000, 640), rand(640)
    y, total, rv, rs = lb.lbscan_block_norm_fwd(rows, w, gate=gate, branch_weight=w, residual=stream, norm_branch=True, return_stats=True)
    one, A, bc, pool = rand(500, 2048), -torch.rand(2048, 16, device="cuda", generator=g), rand(500, 16), rand(500, 2048, 16)
    prompts, conv, before = rand(4, 640, 1000), rand(640, 4), rand(4, 640, 3)
    states = iter([pool.clone() for _ in range(4)])
    conv_states = iter([before.clone() for _ in range(4)])
    return {
        "loss": lambda s: values(lb.lbscan_loss_fwd(x, table, ids, stream=s)),
        "loss gradients": lambda s: values(lb.lbscan_loss_bwd(x, table, ids, lse=lse, dloss=down, stream=s)),
        "loss gradients bf16": lambda s: values(lb.lbscan_loss_bwd(narrow, narrow_table, ids, lse=narrow_lse, dloss=down, stream=s)),
        "norms": lambda s: values(lb.lbscan_block_norm_fwd(rows, w, gate=gate, branch_weight=w, residual=stream, norm_branch=True,
                                                           return_stats=True, stream=s)),
        "norm gradients": lambda s: values(lb.lbscan_block_norm_bwd(rows, w, dout=y, gate=gate, branch_weight=w, total=total, dsum=stream,
                                                                    branch_rstd=rv, stream_rstd=rs, norm_branch=True, stream=s)),
        "step": lambda s: [lb.lbscan_step(one, one, A, bc, bc, next(states), stream=s)],
        "prompt": lambda s: [lb.lbscan_conv1d_prompt(prompts, next(conv_states), conv, stream=s)],
    }


NAMES = ["loss", "loss gradients", "loss gradients bf16", "norms", "norm gradients", "step", "prompt"]


def busy(keep):
    """Some milliseconds of work on the current stream."""
    for _ in range(40):
        keep.add_(1.0)


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_current_stream(lb, name):
    """Blocks of every size that the call may ask for, freed with a copy of them still queued on the current stream."""
    call = calls(lb)[name]
    work = torch.zeros(1 << 26, device="cuda")
    want = [v.clone() for v in call(None)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    s = torch.cuda.Stream()
    sizes = [1 << k for k in range(9, 27)] + [v.numel() * v.element_size() for v in want]
    held = [torch.full((n // 4 + 1,), 3.0, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    busy(work)
    copies = [v.clone() for v in held]
    where = [(v.data_ptr(), v.data_ptr() + v.numel() * 4) for v in held]
    del held
    got = call(s)
    for v in got:
        assert not any(a <= v.data_ptr() < b for a, b in where)
    torch.cuda.synchronize()
    assert all(bool((v == 3.0).all()) for v in copies)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_outputs_that_the_current_stream_still_reads(lb, name):
    """Freed while a copy of them is queued on the current stream, they are not given to the next call."""
    call = calls(lb)[name]
    work = torch.zeros(1 << 26, device="cuda")
    want = [v.clone() for v in call(None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(s)
    s.synchronize()
    busy(work)
    copies = [v.clone() for v in got]
    del got
    again = call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want)) and all(torch.equal(a, b) for a, b in zip(again, want))


def test_a_stream_of_another_device(lb):
    s = torch.cuda.Stream()
    other = types.SimpleNamespace(cuda_stream=s.cuda_stream, stream_id=s.stream_id, device_index=s.device_index + 1,
                                  device_type=s.device_type)
    x, w, y = torch.zeros(4, 16, device="cuda"), torch.zeros(5, 16, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.int64)
    state, conv = torch.zeros(4, 16, 3, device="cuda"), torch.zeros(16, 4, device="cuda")
    A, bc = torch.zeros(16, 3, device="cuda"), torch.zeros(4, 3, device="cuda")
    for call in (lambda: lb.lbscan_loss_fwd(x, w, y, stream=other), lambda: lb.lbscan_loss_bwd(x, w, y, lse=x[:, 0].contiguous(), stream=other),
                 lambda: lb.lbscan_block_norm_fwd(x, stream=other),
                 lambda: lb.lbscan_block_norm_bwd(x, dout=x, stream_rstd=x[:, 0].contiguous(), stream=other),
                 lambda: lb.lbscan_step(x, x, A, bc, bc, state, stream=other), lambda: lb.lbscan_conv1d_step(x, state, conv, stream=other)):
        with pytest.raises(lb.LbscanError, match="device"):
            call()


# ---- outputs and inputs ------------------------------------------------------------------------------------------
def test_outputs_that_share_memory_with_inputs(lb):
    wide = torch.zeros(1, 96, device="cuda")
    out, x = wide[:, 8:40], wide[:, 39:71]                       # one element of both
    clear = torch.zeros(1, 32, device="cuda")
    A, bc, state = torch.zeros(32, 1, device="cuda"), torch.zeros(1, 1, device="cuda"), torch.zeros(1, 32, 1, device="cuda")
    for inputs in ((x, clear, A, bc, bc, state), (clear, x, A, bc, bc, state), (clear, clear, x.view(32, 1), bc, bc, state),
                   (clear, clear, A, out[:, :1], bc, state), (clear, clear, A, bc, out[:, :1], state), (clear, clear, A, bc, bc, x.view(1, 32, 1))):
        with pytest.raises(lb.LbscanError, match="memory"):
            lb.lbscan_step(*inputs, out=out)
    for named in (dict(z=x), dict(Dskip=x[0]), dict(delta_bias=x[0]), dict(conv_weight=x.view(32, 1), conv_state=state[..., :0].contiguous())):
        with pytest.raises(lb.LbscanError, match="memory"):
            lb.lbscan_step(clear, clear, A, bc, bc, state, out=out, **named)
    lb.lbscan_step(wide[:, 40:72], clear, A, bc, bc, state, out=out)      # side by side
    flat = torch.zeros(400, device="cuda")
    p, w, s = flat[:60].view(1, 4, 15), torch.zeros(4, 4, device="cuda"), torch.zeros(1, 4, 3, device="cuda")
    for named in (dict(state=flat[59:71].view(1, 4, 3), weight=w, out=p), dict(state=s, weight=flat[30:46].view(4, 4), out=p),
                  dict(state=s, weight=w, bias=flat[50:54], out=p)):
        with pytest.raises(lb.LbscanError, match="memory"):
            lb.lbscan_conv1d_prompt(flat[100:160].view(1, 4, 15), **named)
    with pytest.raises(lb.LbscanError, match="memory"):
        lb.lbscan_conv1d_prompt(flat[100:160].view(1, 4, 15), s, w, out=flat[159:219].view(1, 4, 15))
    with pytest.raises(lb.LbscanError, match="memory"):
        lb.lbscan_block_norm_fwd(flat[:60].view(4, 15), out=flat[40:100].view(4, 15))
    with pytest.raises(lb.LbscanError, match="memory"):
        lb.lbscan_block_norm_fwd(flat[:60].view(4, 15), flat[160:175], out=flat[170:230].view(4, 15))


# ---- recorded backward passes ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("operator", ["loss", "norms", "embedding"])
def test_recorded_backward_of_leaves_in_use(lb, operator):
    """An eager graph of the same leaves lives on the default stream: the recorded backward pass is refused, and runs once
    the eager graph is gone."""
    from paper_2506_15976_amd import autograd
    x = torch.randn(40, 64, device="cuda", generator=generator(1), requires_grad=True)
    w = torch.randn(90, 64, device="cuda", generator=generator(2), requires_grad=True)
    y = torch.randint(0, 90, (40,), device="cuda", generator=generator(3))

    def run():
        if operator == "loss":
            return autograd.linear_cross_entropy(x, w, y)[0], [x, w]
        if operator == "norms":
            return autograd.block_norm(x), [x]
        return autograd.token_embedding(y, w), [w]
    out, leaves = run()
    down = torch.randn(out.shape, device="cuda", generator=generator(4))
    want = [t.clone() for t in torch.autograd.grad(out, leaves, down)]
    del out
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(run()[0], leaves, down)
    torch.cuda.current_stream().wait_stream(side)
    alive = run()[0]
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(lb.LbscanError, match="captured"):
        with torch.cuda.graph(graph):
            torch.autograd.grad(run()[0], leaves, down)
    del alive, graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(run()[0], leaves, down)
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))

"""Steps, prompts and norms with tensors of more than 2^31 elements: rows at the start, on both sides of the 2^31st element and at the end are
those of a small call, bit for bit (a row is computed in the same way wherever it is)."""
import pytest
import torch

from model_util import generator

pytestmark = pytest.mark.gpu
EDGE = 1 << 31


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


def needs(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GB of device memory")


def places(rows, size):
    """Rows whose values are random and looked at: the first, those around the 2^31st element, the last."""
    k = EDGE // size
    return torch.tensor(sorted({0, 1, k - 1, k, k + 1, rows - 2, rows - 1}), device="cuda")


# norms: every kind of kernel (16 lanes, a wave, several waves, rows that are walked), gate and stream in each
@pytest.mark.parametrize("dim,dtype,gate", [
    (40, torch.float32, True), (768, torch.bfloat16, True), (768, torch.float32, False), (2048, torch.bfloat16, True),
    (8192, torch.bfloat16, False), (10240, torch.bfloat16, True), (20000, torch.float32, False),
])
def test_norms(lb, dim, dtype, gate):
    wide = dtype == torch.float32
    needs(150 if wide else 110)
    n = EDGE // dim + 5000
    at = places(n, dim)
    g = generator(dim)

    def tensor(kind):
        t = torch.zeros(n, dim, device="cuda", dtype=kind)
        t[at] = torch.randn(len(at), dim, device="cuda", generator=g).to(kind)
        return t
    x, residual = tensor(dtype), tensor(torch.float32)
    z = tensor(dtype) if gate else None
    w, bw = torch.randn(dim, device="cuda", generator=g), torch.randn(dim, device="cuda", generator=g)
    options = dict(branch_weight=bw, residual_scale=0.7, norm_branch=True)
    small = lambda t: None if t is None else t[at].contiguous()  # noqa: E731
    y, total, rv, rs = lb.lbscan_block_norm_fwd(x, w, gate=z, residual=residual, return_stats=True, **options)
    want = lb.lbscan_block_norm_fwd(small(x), w, gate=small(z), residual=small(residual), return_stats=True, **options)
    for name, got, ref in zip(("y", "sum", "branch_rstd", "stream_rstd"), (y, total, rv, rs), want):
        assert torch.equal(got[at], ref), name
    assert not y[at[2] - 1].any() and not total[n - 3].any()                # (rows of zeros between them)
    del residual, y
    dout, dsum = tensor(dtype), tensor(torch.float32)
    grads = lb.lbscan_block_norm_bwd(x, w, dout=dout, gate=z, total=total, dsum=dsum, branch_rstd=rv, stream_rstd=rs, **options)
    ref = lb.lbscan_block_norm_bwd(small(x), w, dout=small(dout), gate=small(z), total=want[1], dsum=small(dsum), branch_rstd=want[2],
                                   stream_rstd=want[3], **options)
    for name in ("dx", "dresidual", *(("dgate",) if gate else ())):
        assert torch.equal(grads[name][at], ref[name]), name
        assert not grads[name][at[2] - 1].any() and not grads[name][n - 3].any(), name
    # the weights' gradients are sums of these rows' terms and of zeros, seven terms in another order
    shat = total[at].double() * rs[at, None].double()
    v = x[at].double() * (z[at].double() * torch.sigmoid(z[at].double()) if gate else 1.0)
    for name, terms in (("dweight", dout[at].double() * shat), ("dbranch_weight", ref["dresidual"].double() / 0.7 * v * rv[at, None].double())):
        bound = 16 * 2.0 ** -24 * terms.abs().sum(0)
        assert bool(((grads[name].double() - ref[name].double()).abs() <= bound).all()), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("call", ["step", "large step", "conv step", "prompt"])
def test_pools(lb, call, dtype):
    """A pool of the convolution's states of more than 2^31 elements.  (The large step has a channel a lane.)"""
    D, N, K = 4096, 9 if call == "large step" else 2, 4
    needs(60)
    S = EDGE // (D * (K - 1)) + 3000
    slots = places(S, D * (K - 1)).int()
    if call == "large step":
        slots = torch.cat([slots, torch.arange(2000, 2033, device="cuda", dtype=torch.int32)])
    B = len(slots)
    g = generator(3)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    pool = torch.zeros(S, D, K - 1, device="cuda", dtype=dtype)
    pool[slots.long()] = rand(B, D, K - 1).to(dtype)
    before = pool[slots.long()]
    weight, bias = rand(D, K), rand(D)
    if call.endswith("step") and call != "conv step":
        states = torch.zeros(S, D, N, device="cuda")
        own = rand(B, D, N)
        states[slots.long()] = own
        x, delta, z = (rand(B, D).to(dtype) for _ in range(3))
        rest = (x, delta, -rand(D, N).abs(), rand(B, N).to(dtype), rand(B, N).to(dtype))
        named = dict(Dskip=rand(D), z=z, conv_weight=weight, conv_bias=bias)
        want = lb.lbscan_step(*rest, own, conv_state=before, **named)
        got = lb.lbscan_step(*rest, states, conv_state=pool, slots=slots, **named)
        assert torch.equal(states[slots.long()], own) and not states[S - 3].any()
    elif call == "conv step":
        x = rand(B, D).to(dtype)
        want = lb.lbscan_conv1d_step(x, before, weight, bias)
        got = lb.lbscan_conv1d_step(x, pool, weight, bias, slots=slots)
    else:
        x, lengths = rand(B, D, 37).to(dtype), torch.tensor([37, 0, 1, 2, 3, 20, 36], device="cuda", dtype=torch.int32)
        want = lb.lbscan_conv1d_prompt(x, before, weight, bias, lengths=lengths)
        got = lb.lbscan_conv1d_prompt(x, pool, weight, bias, lengths=lengths, slots=slots)
    assert torch.equal(got, want) and torch.equal(pool[slots.long()], before)
    assert not pool[S - 3].any() and not pool[slots[2] - 1].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,D,L", [(70, 4096, 7500), (5, 40000, 10748), (131100, 4096, 4)])
def test_batches_of_prompts(lb, dtype, B, D, L):
    needs(40)
    assert B * D * L > EDGE > (B - 1) * D * L or B > 70000
    at = sorted({0, EDGE // (D * L) - 1, min(EDGE // (D * L), B - 1), B - 1})
    g = generator(L)
    x = torch.zeros(B, D, L, device="cuda", dtype=dtype)
    state = torch.zeros(B, D, 3, device="cuda", dtype=dtype)
    for b in at:
        x[b], state[b] = torch.randn(D, L, device="cuda", generator=g), torch.randn(D, 3, device="cuda", generator=g)
    lengths = torch.full((B,), L, device="cuda", dtype=torch.int32)
    lengths[at[0]] = L - 1
    weight = torch.randn(D, 4, device="cuda", generator=g)
    own = state[at]
    y = lb.lbscan_conv1d_prompt(x, state, weight, lengths=lengths)
    want = lb.lbscan_conv1d_prompt(x[at], own, weight, lengths=lengths[at])
    assert torch.equal(y[at], want) and torch.equal(state[at], own)
    zeros = [b for b in (1, 2, B // 2, B - 5) if 0 < b < B and b not in at]
    assert zeros and not any(y[b].any() for b in zeros)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("conv", [False, True])
def test_columns_of_a_wide_tensor(lb, dtype, conv):
    """Rows of x, delta, z, B and C that lie so far apart that the last begin behind the 2^31st element."""
    B, D, N = 70, 512, 16
    needs(20)
    pitch = EDGE // (B - 2)
    flat = torch.zeros(B, pitch, device="cuda", dtype=dtype)
    g = generator(5)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    parts = flat[:, -(3 * D + 2 * N):].split([D, D, D, N, N], 1)
    for p in parts:
        p.copy_(rand(*p.shape))
    x, delta, z, Bm, Cm = parts
    A, state, skip = -rand(D, N).abs(), rand(B, D, N), rand(D)
    named = dict(conv_weight=rand(D, 4), conv_state=rand(B, D, 3).to(dtype)) if conv else {}
    again = {k: v.clone() for k, v in named.items()}
    same = state.clone()
    got = lb.lbscan_step(x, delta, A, Bm, Cm, state, skip, z, **named)
    want = lb.lbscan_step(*(t.contiguous() for t in (x, delta)), A, Bm.contiguous(), Cm.contiguous(), same, skip, z.contiguous(), **again)
    assert torch.equal(got, want) and torch.equal(state, same)
    if conv:
        assert torch.equal(named["conv_state"], again["conv_state"])
        before = named["conv_state"].clone()
        assert torch.equal(lb.lbscan_conv1d_step(x, named["conv_state"], named["conv_weight"]),
                           lb.lbscan_conv1d_step(x.contiguous(), before, named["conv_weight"]))
        assert torch.equal(named["conv_state"], before)

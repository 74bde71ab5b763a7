"""Single tokens through the scan and the convolution, and prompts through the convolution with its state, against the
64-bit reference: every width and number of states, pools with padding, slots named twice, ragged prompts, columns of wider
tensors, prompts and steps in turn, graphs, streams."""
import pytest
import torch

import model_reference as ref
from model_util import CONV, STEP, TYPES, generator, guarded
from sequence_util import close, off_by_one, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def step_inputs(B, D, N, dtype, *, K=0, S=None, seed=0, z=True, skip=True, bias=True):
    g = generator(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    S = B if S is None else S
    t = dict(x=rand(B, D).to(dtype), delta=(0.5 * rand(B, D)).to(dtype), A=-16 * torch.rand(D, N, device="cuda", generator=g),
             Bm=rand(B, N).to(dtype), Cm=rand(B, N).to(dtype), state=rand(S, D, N))
    if skip:
        t["Dskip"] = rand(D)
    if z:
        t["z"] = rand(B, D).to(dtype)
    if bias:
        t["delta_bias"] = rand(D) - 2
    if K:
        t.update(conv_state=rand(S, D, K - 1).to(dtype), conv_weight=rand(D, K), conv_bias=rand(D))
    return t


def check_step(lb, t, **options):
    want, state, conv_state = ref.step(**t, **options)
    got = lb.lbscan_step(**t, **options)
    close(got, to_numpy(want), STEP[t["x"].dtype], "y")
    close(t["state"], to_numpy(state), STEP[torch.float32], "state")
    if "conv_state" in t:
        assert torch.equal(t["conv_state"].double().cpu(), conv_state)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,D,N", [(1, 1, 1), (1, 64, 16), (3, 65, 4), (2, 130, 5), (5, 7, 8), (2, 100, 9), (1, 257, 13), (64, 768, 16),
                                   (2, 63, 15)])
def test_step(lb, dtype, B, D, N):
    check_step(lb, step_inputs(B, D, N, TYPES[dtype]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("activation", [True, False])
def test_step_with_its_convolution(lb, dtype, K, activation):
    check_step(lb, step_inputs(3, 70, 16, TYPES[dtype], K=K, seed=K), activation=activation)


@pytest.mark.parametrize("z,skip,bias,softplus", [(False, True, True, True), (True, False, False, True), (False, False, False, False)])
def test_step_without_its_options(lb, z, skip, bias, softplus):
    t = step_inputs(3, 70, 16, torch.float32, z=z, skip=skip, bias=bias)
    if not softplus:
        t["delta"] = t["delta"].abs()
    check_step(lb, t, delta_softplus=softplus)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("slots", [[4, 0, 7], [4, -1, 7], [-1, -1, -1], [3, 3, 0], [2, 8, 2], [-5, 1 << 30, 6]])
def test_pool(lb, dtype, slots):
    """Rows of padding (none of the pool, or an earlier row's) give zeros; all other states stand as they were."""
    t = step_inputs(3, 70, 16, TYPES[dtype], K=4, S=8)
    t["state"], stands = guarded(t["state"])
    t["conv_state"], conv_stands = guarded(t["conv_state"])
    before = t["state"].clone(), t["conv_state"].clone()
    t["slots"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
    y = check_step(lb, t)
    at = ref.places(slots, 3, 8)
    assert stands() and conv_stands()
    for b, s in enumerate(at):
        assert s >= 0 or not y[b].any()
    for s in set(range(8)) - set(at):
        assert torch.equal(t["state"][s], before[0][s]) and torch.equal(t["conv_state"][s], before[1][s])


def test_many_rows_and_slots(lb):
    """More rows than a wave looks through at once, one of them named again at the end."""
    t = step_inputs(300, 33, 16, torch.float32, K=3, S=400)
    slots = torch.randperm(400, device="cuda", generator=generator(1))[:300].to(torch.int32)
    slots[299], slots[150] = slots[7], -1
    check_step(lb, dict(t, slots=slots))


def test_padding_keeps_what_is_not_finite_out(lb):
    t = step_inputs(2, 40, 16, torch.float32, K=4, S=2)
    for k in ("x", "delta", "z", "Bm", "Cm"):
        t[k][1] = float("nan")
    t["state"][1] = float("inf")
    t["slots"] = torch.tensor([0, -1], dtype=torch.int32, device="cuda")
    y = lb.lbscan_step(**t)
    assert torch.isfinite(y).all() and not y[1].any() and torch.isinf(t["state"][1]).all() and torch.isfinite(t["state"][0]).all()


@pytest.mark.parametrize("N", [3, 16])
def test_columns_of_wider_tensors(lb, N):
    t = step_inputs(4, 50, N, torch.bfloat16, K=4)
    wide = torch.randn(4, 2 * 50 + 3, device="cuda").bfloat16()
    proj = torch.randn(4, 2 * N + 7, device="cuda").bfloat16()
    t["x"], t["z"] = wide[:, 1:51], wide[:, 53:]
    t["Bm"], t["Cm"] = proj[:, 7:7 + N], proj[:, 7 + N:]
    check_step(lb, t)


def test_any_alignment(lb):
    t = step_inputs(3, 37, 7, torch.bfloat16, K=4)
    check_step(lb, {k: off_by_one(v) for k, v in t.items()})


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("L", [1, 2, 3, 4, 7, 8, 9, 33, 197])
def test_prompt(lb, dtype, K, L):
    g = generator(L)
    x = torch.randn(3, 41, L, device="cuda", generator=g).to(TYPES[dtype])
    state = torch.randn(3, 41, K - 1, device="cuda", generator=g).to(TYPES[dtype])
    w, b = torch.randn(41, K, device="cuda", generator=g), torch.randn(41, device="cuda", generator=g)
    want, after = ref.conv_prompt(x, state, w, b)
    got = lb.lbscan_conv1d_prompt(x, state, w, b)
    close(got, to_numpy(want), CONV[x.dtype], "y")
    assert torch.equal(state.double().cpu(), after)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L", [5, 40, 203])
@pytest.mark.parametrize("slots", [None, [5, 1, -1, 1, 0, 7]])
def test_ragged_prompts(lb, dtype, L, slots):
    """Lengths from none to all, and beyond both; what stands behind them is not looked at."""
    g = generator(L)
    lengths = [0, 1, 3, L, L + 9, -4]
    K, S = 4, 6 if slots is None else 8
    x = torch.randn(6, 20, L, device="cuda", generator=g).to(TYPES[dtype])
    for b, n in enumerate(lengths):
        x[b, :, max(0, n):] = float("nan")
    state, stands = guarded(torch.randn(S, 20, K - 1, device="cuda", generator=g).to(TYPES[dtype]))
    w = torch.randn(20, K, device="cuda", generator=g)
    want, after = ref.conv_prompt(x, state, w, lengths=lengths, slots=slots, activation=False)
    got = lb.lbscan_conv1d_prompt(x, state, w, activation=False, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                                  slots=None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda"))
    close(got, to_numpy(want), CONV[x.dtype], "y")
    assert torch.equal(state.double().cpu(), after) and stands()


def test_prompts_in_pieces_and_steps(lb):
    """A prompt, a piece of one token, single steps: as the plain convolution of the whole sequence."""
    g = generator(3)
    x = torch.randn(2, 30, 60, device="cuda", generator=g)
    w, b = torch.randn(30, 4, device="cuda", generator=g), torch.randn(30, device="cuda", generator=g)
    want = lb.lbscan_conv1d_fwd(x, w, b)
    state = torch.zeros(2, 30, 3, device="cuda")
    parts = [lb.lbscan_conv1d_prompt(p.contiguous(), state, w, b) for p in x.split([37, 1, 2, 8, 5, 1, 6], 2)[:-1]]
    parts += [lb.lbscan_conv1d_step(x[:, :, t], state, w, b)[..., None] if x[:, :, t].stride(1) == 1 else
              lb.lbscan_conv1d_step(x[:, :, t].contiguous(), state, w, b)[..., None] for t in range(54, 60)]
    close(torch.cat(parts, 2), to_numpy(want), CONV[torch.float32], "pieces")


def test_prompt_and_steps_are_the_scan(lb):
    """Convolution and scan of a prompt, then tokens one by one: as the whole sequence at once."""
    B, D, N, L, cut = 2, 48, 16, 40, 29
    g = generator(9)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, delta, z, Bm, Cm = rand(B, D, L), 0.5 * rand(B, D, L), rand(B, D, L), rand(B, N, L), rand(B, N, L)
    A, skip, bias, w, wb = -8 * torch.rand(D, N, device="cuda", generator=g), rand(D), rand(D) - 2, rand(D, 4), rand(D)
    whole = lb.lbscan_fwd(lb.lbscan_conv1d_fwd(x, w, wb), delta, A, Bm, Cm, skip, z, bias, window=1)
    part = lambda t: t[..., :cut].contiguous()  # noqa: E731
    conv_state = torch.zeros(B, D, 3, device="cuda")
    u = lb.lbscan_conv1d_prompt(part(x), conv_state, w, wb)
    y, state = lb.lbscan_fwd(u, part(delta), A, part(Bm), part(Cm), skip, part(z), bias, window=1, return_state=True)
    close(y, to_numpy(whole[..., :cut]), STEP[torch.float32], "prompt")
    for t in range(cut, L):
        at = lambda v: v[..., t].contiguous()  # noqa: E731
        y = lb.lbscan_step(at(x), at(delta), A, at(Bm), at(Cm), state, skip, at(z), bias, conv_state=conv_state, conv_weight=w,
                           conv_bias=wb)
        close(y, to_numpy(whole[..., t]), STEP[torch.float32], f"token {t}")


def test_empty_sizes(lb):
    for B, D in ((0, 5), (3, 0)):
        t = step_inputs(B, D, 16, torch.float32, K=4)
        assert lb.lbscan_step(**t).shape == (B, D)
    state = torch.randn(2, 5, 3, device="cuda")
    before = state.clone()
    assert lb.lbscan_conv1d_prompt(torch.empty(2, 5, 0, device="cuda"), state, torch.ones(5, 4, device="cuda")).shape == (2, 5, 0)
    assert torch.equal(state, before)
    # a pool of no rows: every row is padding
    t = step_inputs(2, 5, 16, torch.float32, K=4, S=0)
    assert not lb.lbscan_step(**t, slots=torch.zeros(2, dtype=torch.int32, device="cuda")).any()


def test_more_rows_than_the_grid_has(lb):
    B = 70000
    t = step_inputs(B, 3, 2, torch.float32, K=2)
    rows = [0, 65534, 65535, 65536, B - 1]
    some = {k: v[rows].clone() if v.shape[0] == B else v for k, v in t.items()}
    want, state, _ = ref.step(**some)
    got = lb.lbscan_step(**t)
    close(got[rows], to_numpy(want), STEP[torch.float32], "y")
    close(t["state"][rows], to_numpy(state), STEP[torch.float32], "state")
    x = torch.randn(B, 2, 3, device="cuda")
    conv_state, w = torch.randn(B, 2, 1, device="cuda"), torch.randn(2, 2, device="cuda")
    want, after = ref.conv_prompt(x[rows], conv_state[rows], w)
    close(lb.lbscan_conv1d_prompt(x, conv_state, w)[rows], to_numpy(want), CONV[torch.float32], "y")
    assert torch.equal(conv_state[rows].double().cpu(), after)


def test_pool_beyond_2_31_elements(lb):
    """A pool of 2^29 + states: 9 GB, offsets of more than 32 bits."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB of device memory")
    D, N = 4096, 16
    S = (1 << 31) // (D * N) + 3
    pool = torch.zeros(S, D, N, device="cuda")
    t = step_inputs(2, D, N, torch.float32)
    small = dict(t, state=t["state"].clone())
    pool[S - 1], pool[0] = t["state"][0], t["state"][1]
    want = lb.lbscan_step(**small)
    got = lb.lbscan_step(**dict(t, state=pool), slots=torch.tensor([S - 1, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want) and torch.equal(pool[S - 1], small["state"][0]) and torch.equal(pool[0], small["state"][1])
    del pool
    torch.cuda.empty_cache()


def test_replayed_in_a_graph(lb):
    """Tokens of a captured step, slots changed between the replays: as eager steps."""
    t = step_inputs(4, 64, 16, torch.bfloat16, K=4, S=6)
    t["slots"] = torch.tensor([0, 3, 5, -1], dtype=torch.int32, device="cuda")
    eager = {k: v.clone() for k, v in t.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lb.lbscan_step(**{k: v.clone() for k, v in t.items()})
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lb.lbscan_step(**t)
    for k in range(4):
        x = torch.randn(4, 64, device="cuda").bfloat16()
        slots = torch.tensor([[0, 3, 5, -1], [0, 3, 5, 1], [2, 2, 5, 1], [5, 3, 0, -1]][k], dtype=torch.int32, device="cuda")
        for d in (t, eager):
            d["x"].copy_(x)
            d["slots"].copy_(slots)
        graph.replay()
        want = lb.lbscan_step(**eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(t["state"], eager["state"]) and torch.equal(t["conv_state"], eager["conv_state"])


def test_on_a_named_stream(lb):
    t = step_inputs(4, 64, 16, torch.float32, K=4)
    other = {k: v.clone() for k, v in t.items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = lb.lbscan_step(**t, stream=side)
    side.synchronize()
    assert torch.equal(got, lb.lbscan_step(**other)) and torch.equal(t["state"], other["state"])


def test_overwritten_tensors_count_their_versions(lb):
    t = step_inputs(2, 8, 4, torch.float32, K=2)
    versions = t["state"]._version, t["conv_state"]._version
    out = torch.empty_like(t["x"])
    lb.lbscan_step(**t, out=out)
    assert t["state"]._version > versions[0] and t["conv_state"]._version > versions[1] and out._version > 0
    t["state"].requires_grad_(True)
    with pytest.raises(lb.LbscanError):
        lb.lbscan_step(**t)
    with torch.no_grad():
        lb.lbscan_step(**t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,D,N,K", [(300, 450, 16, 4), (300, 450, 9, 1), (300, 450, 13, 2), (300, 449, 16, 3), (300, 450, 16, 0), (600, 450, 8, 0),
                                     (600, 450, 5, 4), (1100, 450, 4, 0), (1100, 300, 3, 4), (2100, 20, 16, 4), (2100, 65, 12, 0)])
def test_large_steps(lb, dtype, B, D, N, K):
    """The launches of large calls: rows and channels that no wave divides, a pool with padding and a slot named twice."""
    t = step_inputs(B, D, N, TYPES[dtype], K=K, S=B + 7)
    slots = torch.randperm(B + 7, device="cuda", generator=generator(3))[:B].int()
    slots[B // 2], slots[B - 3], slots[5] = -1, slots[1], B + 7
    before = {k: t[k].clone() for k in ("state", "conv_state") if k in t}
    check_step(lb, t, slots=slots)
    free = torch.ones(B + 7, dtype=torch.bool, device="cuda")
    free[slots[(slots >= 0) & (slots < B + 7)].long()] = False
    for k, v in before.items():
        assert torch.equal(t[k][free], v[free]), k

"""Gated linear recurrence on the GPU against the 64-bit reference: every family of launch shapes, both directions,
packed sequences, states in and out, gates that are closed, and what must not leak out of a masked past."""
import ctypes

import numpy as np
import pytest
import torch

import sequence_reference as ref
from sequence_util import GATED, TYPES, close, off_by_one, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def make(B, D, L, dtype="fp32", seed=0, starts=False, state=True):
    g = torch.Generator().manual_seed(1000 * seed + L)
    dt = TYPES[dtype]
    t = {k: torch.randn(B, D, L, generator=g).to(dt).cuda() for k in ("x", "gate_a", "gate_x")}
    open_gate = torch.empty(D).uniform_(0.9, 0.999, generator=g)
    t["decay"] = torch.log(torch.expm1(-torch.log(open_gate) / 8)).cuda()
    if starts:
        t["starts"] = (torch.rand(B, L, generator=g) < min(0.5, 5.0 / L)).cuda()
    if state:
        t["h0"] = torch.randn(B, D, generator=g).cuda()
    more = dict(dout=torch.randn(B, D, L, generator=g).to(dt).cuda(), dhT=torch.randn(B, D, generator=g).cuda())
    return t, more


def reference(t, more, reverse):
    n = {k: to_numpy(v) for k, v in t.items()}
    keys = dict(starts=n.get("starts"), reverse=reverse, h0=n.get("h0"))
    y, h, _ = ref.gated_fwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], **keys)
    dhT = to_numpy(more["dhT"]) if more.get("dhT") is not None else None
    return y, h, ref.gated_bwd(n["x"], n["gate_a"], n["gate_x"], n["decay"], to_numpy(more["dout"]), dhT=dhT, **keys)


def check(lb, t, more, dtype, reverse=False):
    y, hT, want = reference(t, more, reverse)
    tol = GATED[dtype]
    saved = lb.lbscan_gated_saved_state(t["x"], reverse=reverse)
    got, gT = lb.lbscan_gated_fwd(**t, reverse=reverse, return_state=True, saved_state=saved)
    close(got, y, tol, "y")
    close(gT, hT, GATED["fp32"], "hT")
    first = None
    for keep in (saved, None):
        g = lb.lbscan_gated_bwd(**t, **more, reverse=reverse, saved_state=keep)
        for k, v in g.items():
            close(v, want[k], GATED["fp32"] if k in ("ddecay", "dh0") else tol, k)
        if first is None:
            first = g
        else:                                    # computed again or kept: the same states
            assert all(torch.equal(first[k], g[k]) for k in g)


LENGTHS = [1, 2, 7, 8, 9, 31, 63, 64, 65, 128, 197, 255, 256, 257, 511, 512, 513, 1023, 1025, 2050, 4099, 9001]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L", LENGTHS)
def test_lengths(lb, L, reverse, dtype):
    t, more = make(2, 5 if L < 2000 else 3, L, dtype, seed=1)
    check(lb, t, more, dtype, reverse)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L", [1, 5, 8, 60, 100, 197, 300, 600, 1500, 9001])
def test_packed_sequences(lb, L, reverse, dtype):
    t, more = make(3, 3, L, dtype, seed=2, starts=True)
    check(lb, t, more, dtype, reverse)


# few long rows, which are cut into pieces that several blocks take
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L,starts", [(33000, False), (40001, True)])
def test_cut_rows(lb, L, starts, reverse, dtype):
    t, more = make(1, 3, L, dtype, seed=19, starts=starts)
    assert lb.load().lbscan_gated_workspace_bytes(ctypes.byref(lb.LbscanGatedArgs(1, 3, L, int(dtype == "bf16"))), 0) > 0
    check(lb, t, more, dtype, reverse)


# rows enough that a row is not cut: one wave, four waves, sixteen waves a row, several tiles each
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,D,L", [(17, 513, 1300), (2, 150, 3300), (1, 300, 17000)])
@pytest.mark.parametrize("starts", [False, True])
def test_whole_rows(lb, B, D, L, dtype, starts):
    t, more = make(B, D, L, dtype, seed=3, starts=starts)
    check(lb, t, more, dtype, reverse=starts)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_without_states(lb, dtype):
    for L in (3, 50, 700):
        t, more = make(2, 4, L, dtype, seed=4, state=False)
        del more["dhT"]
        y, _, want = reference(t, more, False)
        close(lb.lbscan_gated_fwd(**t), y, GATED[dtype], "y")
        g = lb.lbscan_gated_bwd(**t, **more)
        assert "dh0" not in g
        for k, v in g.items():
            close(v, want[k], GATED["fp32"] if k == "ddecay" else GATED[dtype], k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("L", [5, 24, 197, 1030])
def test_any_alignment(lb, L, dtype):
    t, more = make(2, 3, L, dtype, seed=5, starts=True)
    moved = {k: off_by_one(v) for k, v in t.items()}
    shifted = {k: off_by_one(v) for k, v in more.items()}
    out = off_by_one(torch.zeros_like(t["x"]))
    assert torch.equal(lb.lbscan_gated_fwd(**moved, out=out), lb.lbscan_gated_fwd(**t))
    a, b = lb.lbscan_gated_bwd(**moved, **shifted), lb.lbscan_gated_bwd(**t, **more)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_nothing_is_written_beside_the_outputs(lb):
    for dtype in ("fp32", "bf16"):
        for L in (3, 9, 197, 515):
            t, _ = make(2, 3, L, dtype, seed=6)
            room = torch.full((2 * 3 * L + 64,), 7.0, dtype=TYPES[dtype], device="cuda")
            for reverse in (False, True):
                lb.lbscan_gated_fwd(**t, out=room[32:-32].view(2, 3, L), reverse=reverse)
                assert bool((room[:32] == 7).all()) and bool((room[-32:] == 7).all())


def test_empty(lb):
    for B, D, L in ((0, 3, 5), (2, 0, 5), (2, 3, 0)):
        t, more = make(B, D, L)
        y, hT = lb.lbscan_gated_fwd(**t, return_state=True)
        assert y.shape == (B, D, L) and torch.equal(hT, t["h0"])
        g = lb.lbscan_gated_bwd(**t, **more)
        assert torch.equal(g["dh0"], more["dhT"]) and not g["ddecay"].any()


@pytest.mark.parametrize("L", [4, 40, 600])
def test_closed_and_open_gates(lb, L):
    """sqrt(1 - a^2) has no derivative where the gate is closed (a = 1); the gradients have limits."""
    t, more = make(2, 6, L, seed=7)
    t["gate_a"][:, 0] = -200.0
    t["gate_a"][:, 1] = 200.0
    t["gate_a"][:, 2, ::2] = -30.0
    t["gate_x"][:, 3] = -200.0
    t["gate_x"][:, 4] = 200.0
    t["decay"][5] = -200.0
    y, hT, want = reference(t, more, False)
    got = lb.lbscan_gated_fwd(**t)
    g = lb.lbscan_gated_bwd(**t, **more)
    for c in range(6):                           # (channel by channel: their scales differ)
        close(got[:, c], y[:, c], GATED["fp32"], f"y {c}")
        for k in ("dx", "dgate_a", "dgate_x"):
            w = want[k][:, c]
            if np.abs(w).max() < 1e-30:
                assert float(g[k][:, c].abs().max()) < 1e-30, (k, c)
            else:
                close(g[k][:, c], w, GATED["fp32"], f"{k} {c}")
    close(g["ddecay"], want["ddecay"], GATED["fp32"], "ddecay")


@pytest.mark.parametrize("decay", [-60.0, -4.1, -3.3, -2.5, 0.0, 5.0, 40.0])
def test_decay_range(lb, decay):
    t, more = make(2, 3, 100, seed=8)
    t["decay"][:] = decay
    check(lb, t, more, "fp32")


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L,cut", [(6, 3), (50, 20), (197, 100), (700, 333), (9001, 4500), (40001, 23456)])
def test_a_start_keeps_the_past_out(lb, L, cut, reverse):
    """NaN and infinities before a start, in tokens and in the state, reach nothing behind it, nor do gradients
    behind a start reach what is before it."""
    t, more = make(1, 2, L, seed=9)
    t["starts"] = torch.zeros(1, L, dtype=torch.bool, device="cuda")
    t["starts"][0, cut] = True
    past = slice(cut + 1, None) if reverse else slice(0, cut)
    rest = slice(0, cut + 1) if reverse else slice(cut, None)
    clean = lb.lbscan_gated_fwd(**t, reverse=reverse, return_state=True)
    clean_g = lb.lbscan_gated_bwd(**t, **more, reverse=reverse)
    bad = {k: v.clone() for k, v in t.items()}
    bad["x"][0, 0, past] = float("nan")
    bad["x"][0, 1, past] = float("inf")
    bad["h0"][:] = float("nan")
    y, hT = lb.lbscan_gated_fwd(**bad, reverse=reverse, return_state=True)
    assert torch.equal(y[..., rest], clean[0][..., rest]) and torch.equal(hT, clean[1])
    assert not torch.isfinite(y[..., past]).any()
    g = lb.lbscan_gated_bwd(**bad, **more, reverse=reverse)
    for k in ("dx", "dgate_a", "dgate_x"):
        assert torch.equal(g[k][..., rest], clean_g[k][..., rest]), k
    # gradients of the other sequence
    late = {k: v.clone() for k, v in more.items()}
    late["dout"][..., rest] = float("nan")
    late["dhT"][:] = float("inf")
    g = lb.lbscan_gated_bwd(**t, **late, reverse=reverse)
    for k in ("dx", "dgate_a", "dgate_x"):
        assert torch.equal(g[k][..., past], clean_g[k][..., past]), k
    assert torch.equal(g["dh0"], clean_g["dh0"])


def test_packed_equals_apart(lb):
    t, more = make(1, 4, 300, seed=10)
    t["starts"] = torch.zeros(1, 300, dtype=torch.uint8, device="cuda")
    t["starts"][0, 130] = 255
    y = lb.lbscan_gated_fwd(**t)
    parts = []
    for a, b, h0 in ((0, 130, t["h0"]), (130, 300, None)):
        s = {k: t[k][..., a:b].contiguous() for k in ("x", "gate_a", "gate_x")}
        parts.append(lb.lbscan_gated_fwd(**s, decay=t["decay"], h0=h0))
    close(y, to_numpy(torch.cat(parts, -1)), GATED["fp32"], "y")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_steps_equal_the_prompt(lb, dtype):
    t, _ = make(3, 70, 12, dtype, seed=11, starts=True)
    y, hT, _ = reference(t, dict(dout=t["x"]), False)
    state = t["h0"].clone()
    where = state.data_ptr()
    for k in range(12):
        out = lb.lbscan_gated_step(*(t[n][..., k].contiguous() for n in ("x", "gate_a", "gate_x")), t["decay"], state,
                                   starts=t["starts"][:, k].contiguous())
        close(out, y[..., k], GATED[dtype], f"token {k}")
    assert state.data_ptr() == where
    close(state, hT, GATED["fp32"], "state")


@pytest.mark.parametrize("B,D,L", [(2, 3, 5), (2, 3, 50), (1, 300, 3000), (1, 3, 9001), (1, 3, 50000)])
def test_state_in_place(lb, B, D, L):
    """hT may be h0, also where a row is cut and every piece reads the state that enters."""
    from paper_2506_15976_amd import binding
    t, _ = make(B, D, L, seed=12)
    y, hT = lb.lbscan_gated_fwd(**t, return_state=True)
    state, out = t["h0"].clone(), torch.empty_like(t["x"])
    a = lb.LbscanGatedArgs(B, D, L, 0, 0, 8.0, t["x"].data_ptr(), t["gate_a"].data_ptr(), t["gate_x"].data_ptr(),
                           t["decay"].data_ptr(), None, state.data_ptr(), out.data_ptr(), state.data_ptr())
    a.workspace_bytes = lb.load().lbscan_gated_workspace_bytes(ctypes.byref(a), binding.WS_FWD)
    ws = torch.empty(a.workspace_bytes + 4, dtype=torch.uint8, device="cuda")
    a.workspace = ws.data_ptr()
    assert lb.load().lbscan_gated_fwd(ctypes.byref(a), binding._stream(None)) == 0
    assert torch.equal(out, y) and torch.equal(state, hT)


def test_pieces_add_up(lb):
    t, _ = make(1, 4, 1000, seed=13)
    whole, hT = lb.lbscan_gated_fwd(**t, return_state=True)
    h, parts = t["h0"], []
    for a, b in ((0, 7), (7, 600), (600, 1000)):
        s = {k: t[k][..., a:b].contiguous() for k in ("x", "gate_a", "gate_x")}
        y, h = lb.lbscan_gated_fwd(**s, decay=t["decay"], h0=h, return_state=True)
        parts.append(y)
    close(torch.cat(parts, -1), to_numpy(whole), GATED["fp32"], "y")
    close(h, to_numpy(hT), GATED["fp32"], "hT")


@pytest.mark.parametrize("packed", [False, True])
def test_autograd(lb, packed):
    from paper_2506_15976_amd.autograd import gated_linear_recurrence
    t, more = make(2, 5, 130, seed=14, starts=packed)
    y, hT, want = reference(t, more, True)
    names = ("x", "gate_a", "gate_x", "decay", "h0")
    for k in names:
        t[k].requires_grad_(True)
    got, gT = gated_linear_recurrence(**t, reverse=True, return_state=True)
    close(got, y, GATED["fp32"], "y")
    grads = torch.autograd.grad((got, gT), [t[k] for k in names], (more["dout"], more["dhT"]))
    for g, k in zip(grads, ("dx", "dgate_a", "dgate_x", "ddecay", "dh0")):
        close(g, want[k], GATED["fp32"], k)
    # transposed inputs, and a loss on the state alone
    x = t["x"].detach().transpose(1, 2).contiguous().transpose(1, 2).requires_grad_(True)
    _, gT = gated_linear_recurrence(x, t["gate_a"], t["gate_x"], t["decay"], starts=t.get("starts"), h0=t["h0"], return_state=True)
    dx, = torch.autograd.grad(gT, x, more["dhT"])
    _, _, want = reference(t, dict(dout=torch.zeros_like(more["dout"]), dhT=more["dhT"]), False)
    close(dx, want["dx"], GATED["fp32"], "dx of hT")


def test_gradient_against_differences(lb):
    """Directional derivatives of the kernel's own forward pass."""
    t, more = make(2, 40, 150, seed=15)
    g = lb.lbscan_gated_bwd(**t, **more)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def loss(**k):
        y, h = lb.lbscan_gated_fwd(**{**t, **k}, return_state=True)
        return float((y.double() * more["dout"]).sum() + (h.double() * more["dhT"]).sum())

    for name, key in (("x", "dx"), ("gate_a", "dgate_a"), ("gate_x", "dgate_x"), ("decay", "ddecay"), ("h0", "dh0")):
        d = torch.randn(t[name].shape, device="cuda", generator=gen)
        eps = 1e-2
        want = (loss(**{name: t[name] + eps * d}) - loss(**{name: t[name] - eps * d})) / (2 * eps)
        got = float((g[key].double() * d).sum())
        # third derivatives times eps^2 / 6, rounding of the loss (12000 terms) over 2 eps
        scale = float((g[key].double() ** 2).sum().sqrt())
        assert abs(got - want) <= 2e-3 * (abs(want) + scale), (name, got, want)


def test_same_bits_every_time(lb):
    t, more = make(4, 130, 1111, seed=16)
    a, b = (lb.lbscan_gated_bwd(**t, **more) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_another_stream(lb):
    t, more = make(2, 64, 3000, seed=17)
    want, g = lb.lbscan_gated_fwd(**t), lb.lbscan_gated_bwd(**t, **more)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, h = lb.lbscan_gated_fwd(**t, stream=s), lb.lbscan_gated_bwd(**t, **more, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and all(torch.equal(h[k], g[k]) for k in g)


def test_step_in_a_graph(lb):
    t, _ = make(2, 64, 1, seed=18)
    args = [t[n][..., 0].contiguous() for n in ("x", "gate_a", "gate_x")]
    state, out = t["h0"].clone(), torch.empty_like(args[0])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        lb.lbscan_gated_step(*args, t["decay"], state, out=out)
    s.synchronize()
    state.copy_(t["h0"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lb.lbscan_gated_step(*args, t["decay"], state, out=out)
    eager = t["h0"].clone()
    state.copy_(t["h0"])
    for _ in range(3):
        graph.replay()
        want = lb.lbscan_gated_step(*args, t["decay"], eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(state, eager)

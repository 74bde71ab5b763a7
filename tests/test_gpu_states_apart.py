"""States that steps and prompts write share no memory with what the call reads or writes besides; memory side by side, or between
the rows of a wider tensor, is none of it."""
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


B, D, N, K = 2, 32, 4, 4


def given():
    g = generator(1)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    return dict(x=rand(B, D), delta=rand(B, D), A=-rand(D, N).abs(), Bm=rand(B, N), Cm=rand(B, N), state=rand(B, D, N), Dskip=rand(D),
                z=rand(B, D), delta_bias=rand(D), conv_state=rand(B, D, K - 1), conv_weight=rand(D, K), conv_bias=rand(D),
                slots=torch.arange(B, device="cuda", dtype=torch.int32))


INPUTS = ("x", "delta", "A", "Bm", "Cm", "Dskip", "z", "delta_bias", "conv_weight", "conv_bias", "slots")


def at_the_end(t, shape, dtype=torch.float32):
    """A tensor whose first element is the last of t."""
    n = torch.Size(shape).numel()
    flat = torch.zeros(t.numel() + n, device="cuda")
    t.set_(flat[:t.numel()].view(t.shape))
    return flat[t.numel() - 1:t.numel() - 1 + n].view(shape).view(dtype)


@pytest.mark.parametrize("written", ["state", "conv_state"])
@pytest.mark.parametrize("name", INPUTS)
def test_a_step_refuses_inputs_in_its_states(lb, written, name):
    t = given()
    t[name] = at_the_end(t[written], t[name].shape, t[name].dtype)
    with pytest.raises(lb.LbscanError, match=f"^{written} must not.* {name}$"):
        lb.lbscan_step(**t)


def test_a_step_refuses_states_in_each_other(lb):
    t = given()
    t["conv_state"] = at_the_end(t["state"], t["conv_state"].shape)
    with pytest.raises(lb.LbscanError, match="memory"):
        lb.lbscan_step(**t)
    t["conv_state"] = t["state"].view(-1)[:B * D * (K - 1)].view(B, D, K - 1)
    with pytest.raises(lb.LbscanError, match="memory"):
        lb.lbscan_step(**t)


@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("name", ["x", "weight", "bias", "lengths", "slots"])
def test_a_prompt_refuses_inputs_in_its_state(lb, single, name):
    if single and name == "lengths":
        return
    t = dict(x=torch.ones(B, D, device="cuda") if single else torch.ones(B, D, 9, device="cuda"), state=torch.zeros(B, D, K - 1, device="cuda"),
             weight=torch.ones(D, K, device="cuda"), bias=torch.ones(D, device="cuda"), slots=torch.arange(B, device="cuda", dtype=torch.int32))
    if not single:
        t["lengths"] = torch.full((B,), 9, device="cuda", dtype=torch.int32)
    t[name] = at_the_end(t["state"], t[name].shape, t[name].dtype)
    with pytest.raises(lb.LbscanError, match=f"^state must not.* {name}$"):
        (lb.lbscan_conv1d_step if single else lb.lbscan_conv1d_prompt)(**t)


def test_side_by_side_and_between_rows(lb):
    """Everything in one piece of memory, one behind the other; states and output between the rows of a tensor that x is columns of."""
    t = given()
    want = [lb.lbscan_step(**{k: v.clone() for k, v in t.items()})]
    flat, at = torch.zeros(sum(v.numel() for v in t.values()) + B * D, device="cuda"), 0
    for k, v in t.items():
        part = flat[at:at + v.numel()].view(v.dtype).view(v.shape)
        part.copy_(v)
        t[k], at = part, at + v.numel()
    assert torch.equal(lb.lbscan_step(**t, out=flat[at:].view(B, D)), want[0])
    t = given()
    room = B * D * N + B * D
    wide = torch.zeros(B, D + room, device="cuda")
    wide[:, :D] = t["x"]
    t["x"] = wide[:, :D]
    state = wide[0, D:D + B * D * N].view(B, D, N)
    state.copy_(t["state"])
    got = lb.lbscan_step(**{**t, "state": state}, out=wide[0, -B * D:].view(B, D))
    assert torch.equal(got, want[0])
    with pytest.raises(lb.LbscanError, match="memory"):                 # one element of the second row of x
        lb.lbscan_step(**t, out=wide.view(-1)[D + room + 1 - B * D:D + room + 1].view(B, D))
    with pytest.raises(lb.LbscanError, match="memory"):                 # one of the first
        lb.lbscan_step(**t, out=wide.view(-1)[D - 1:D - 1 + B * D].view(B, D))

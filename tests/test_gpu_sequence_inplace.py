"""What the operators around the scan write in place is seen by autograd: version counters, and tensors that
require gradients."""
import pytest
import torch

from paper_2506_15976_amd.binding import EINVAL, LbscanError

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def rows(*shape):
    return torch.randn(*shape, device="cuda")


def refused(f, *args, **k):
    with pytest.raises(LbscanError) as e:
        f(*args, **k)
    assert e.value.code == EINVAL and "requires grad" in str(e.value)


def test_a_step_over_a_saved_state(lb):
    """The state that entered a recurrence is needed by its backward pass, which must not run with another one."""
    from paper_2506_15976_amd.autograd import gated_linear_recurrence
    u, one, decay, state = rows(2, 3, 40).requires_grad_(True), rows(2, 3), rows(3), rows(2, 3)
    y = gated_linear_recurrence(u, u, u, decay, h0=state)
    lb.lbscan_gated_step(one, one, one, decay, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_an_output_over_a_saved_tensor(lb):
    from paper_2506_15976_amd.autograd import layer_norm
    x = rows(6, 40)
    w = torch.ones(40, device="cuda", requires_grad=True)
    y = layer_norm(x, w)
    lb.lbscan_norm_fwd(rows(6, 40), out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_versions(lb):
    u, one, decay, state = rows(2, 3, 40), rows(2, 3), rows(3), rows(2, 3)
    saved = lb.lbscan_gated_saved_state(rows(2, 3, 40000))
    table, ids = rows(5, 8), torch.zeros(7, dtype=torch.int64, device="cuda")
    long = rows(2, 3, 40000)
    calls = [(lambda out: lb.lbscan_gated_fwd(u, u, u, decay, out=out), torch.empty_like(u)),
             (lambda out: lb.lbscan_gated_step(one, one, one, decay, rows(2, 3), out=out), torch.empty_like(one)),
             (lambda out: lb.lbscan_gated_step(one, one, one, decay, out), state),
             (lambda out: lb.lbscan_gated_fwd(long, long, long, decay, saved_state=out), saved),
             (lambda out: lb.lbscan_norm_fwd(u, out=out), torch.empty_like(u)),
             (lambda out: lb.lbscan_embed_fwd(ids, table, out=out), rows(7, 8))]
    for k, (call, out) in enumerate(calls):
        before = out._version
        call(out)
        assert out._version > before, k
    # what a call only reads keeps its version, and so does what a refused call would have written
    assert [v._version for v in (u, one, decay, table, ids, long)] == [0] * 6
    out = torch.empty_like(u)
    with pytest.raises(LbscanError):
        lb.lbscan_gated_fwd(u, u, u, decay, rate=-1.0, out=out)
    assert out._version == 0


def test_tensors_that_require_gradients(lb):
    u, one, decay, state = rows(2, 3, 40), rows(2, 3), rows(3), rows(2, 3)
    table, ids = rows(5, 8), torch.zeros(7, dtype=torch.int64, device="cuda")
    keep = state.clone().requires_grad_(True)
    refused(lb.lbscan_gated_step, one, one, one, decay, keep)
    refused(lb.lbscan_gated_step, one, one, one, decay, state, out=rows(2, 3).requires_grad_(True))
    refused(lb.lbscan_gated_fwd, u, u, u, decay, out=rows(2, 3, 40).requires_grad_(True))
    refused(lb.lbscan_norm_fwd, u, out=rows(2, 3, 40).requires_grad_(True))
    refused(lb.lbscan_embed_fwd, ids, table, out=rows(7, 8).requires_grad_(True))
    # without gradients they are tensors like others
    with torch.no_grad():
        want = state.clone()
        lb.lbscan_gated_step(one, one, one, decay, want)
        lb.lbscan_gated_step(one, one, one, decay, keep)
    assert torch.equal(keep, want)


def test_inference_tensors(lb):
    """They have no version."""
    one, decay, state = rows(2, 3), rows(3), rows(2, 3)
    want, after = lb.lbscan_gated_step(one, one, one, decay, state.clone()), state.clone()
    lb.lbscan_gated_step(one, one, one, decay, after)
    with torch.inference_mode():
        s, out = state.clone(), torch.empty_like(one)
        lb.lbscan_gated_step(one, one, one, decay, s, out=out)
    assert torch.equal(out, want) and torch.equal(s, after)

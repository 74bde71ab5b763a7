"""The scan and its convolution on a stream that the caller names: no memory of another stream's pending work."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


NAMES = ["fwd", "fwd with states", "bwd", "bidir", "columns", "conv", "conv gradients"]


def calls(lb):
    """name -> a call that takes the stream and returns every tensor it made."""
    from gpu_util import fwd_inputs, to_device
    from paper_2506_15976_amd.inputs import make_inputs
    s = to_device(make_inputs(1, 64, 16, 3000, seed=55, with_dout=True), "fp32")      # long rows: scratch in use
    t, dout = fwd_inputs(s), s["dout"]
    h0 = torch.randn(1, 64, 16, device="cuda")
    weight, bias = torch.randn(64, 4, device="cuda"), torch.randn(64, device="cuda")

    def training(stream):
        saved = lb.lbscan_saved_state(t["x"], t["A"], window=4, stream=stream)
        out = lb.lbscan_fwd(**t, window=4, h0=h0, return_state=True, saved_state=saved, stream=stream)
        g = lb.lbscan_bwd(**t, dout=dout, window=4, h0=h0, saved_state=saved, stream=stream)
        return [v for v in (saved, *out, *g.values()) if v is not None]

    other = dict(t, z=None)
    return {
        "fwd": lambda s: [lb.lbscan_fwd(**t, window=4, stream=s)],
        "fwd with states": training,
        "bwd": lambda s: [v for v in lb.lbscan_bwd(**t, dout=dout, window=4, stream=s).values() if v is not None],
        "bidir": lambda s: [lb.lbscan_bidir_fwd(t, other, stream=s)],
        "columns": lambda s: [lb.lbscan_fwd(**t, window=4, grid=(50, 60), stream=s)],
        "conv": lambda s: [lb.lbscan_conv1d_fwd(t["x"], weight, bias, stream=s)],
        "conv gradients": lambda s: list(lb.lbscan_conv1d_bwd(t["x"], weight, bias, dy=dout, stream=s).values()),
    }


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_current_stream(lb, name):
    """Blocks of every size that the call may ask for, freed with a copy of them still queued on the current stream."""
    call = calls(lb)[name]
    work = torch.zeros(1 << 26, device="cuda")
    made = [v.clone() for v in call(None)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    s = torch.cuda.Stream()
    sizes = [1 << k for k in range(9, 26)] + [v.numel() * v.element_size() for v in made]
    held = [torch.full((n // 4 + 1,), 3.0, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(40):                          # some milliseconds
        work.add_(1.0)
    copies = [v.clone() for v in held]
    where = [(v.data_ptr(), v.data_ptr() + v.numel() * 4) for v in held]
    del held
    got = call(s)
    for v in got:
        assert not any(a <= v.data_ptr() < b for a, b in where)
    torch.cuda.synchronize()
    assert all(bool((v == 3.0).all()) for v in copies)
    # (sums by atomics: not the same bits every time)
    for a, b in zip(got, made):
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-4 * float(b.abs().max()))


@pytest.mark.parametrize("name", NAMES)
def test_outputs_that_the_current_stream_still_reads(lb, name):
    """Freed while a copy of them is queued on the current stream, they are not given to the next call."""
    call = calls(lb)[name]
    work = torch.zeros(1 << 26, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(s)
    s.synchronize()
    want = [v.clone() for v in got]
    torch.cuda.synchronize()
    for _ in range(40):
        work.add_(1.0)
    copies = [v.clone() for v in got]
    sizes = [v.shape for v in got]
    del got
    with torch.cuda.stream(s):
        over = [torch.full(n, 5.0, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want))
    del over

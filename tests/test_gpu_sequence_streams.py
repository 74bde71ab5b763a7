"""The operators around the scan on a stream that the caller names: no memory of another stream's pending work."""
import types

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


def calls(lb):
    """name -> a call that takes the stream and returns every tensor it made."""
    g = torch.Generator(device="cuda").manual_seed(1)

    def rand(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    x, decay, h0 = rand(2, 64, 9000), rand(64), rand(2, 64)
    rows, w = rand(3000, 640), rand(640)
    y, total, mean, rstd = lb.lbscan_norm_fwd(rows, w, residual=rows, return_stats=True)
    table, ids = rand(5000, 300), torch.randint(0, 5000, (9000,), device="cuda", generator=g)
    dout = rand(9000, 300)
    one = rand(512, 2048)
    states = iter([one.clone() for _ in range(4)])

    def values(r):
        return [v for v in (r.values() if isinstance(r, dict) else r) if v is not None]

    def training(s):
        saved = lb.lbscan_gated_saved_state(x, stream=s)
        out = lb.lbscan_gated_fwd(x, x, x, decay, h0=h0, return_state=True, saved_state=saved, stream=s)
        return [saved, *out, *values(lb.lbscan_gated_bwd(x, x, x, decay, dout=x, h0=h0, saved_state=saved, stream=s))]

    return {
        "gated": training,
        "gated again": lambda s: values(lb.lbscan_gated_bwd(x, x, x, decay, dout=x, stream=s)),
        "gated cut": lambda s: [lb.lbscan_gated_fwd(x.view(1, 8, -1), x.view(1, 8, -1), x.view(1, 8, -1), decay[:8], stream=s)],
        "step": lambda s: [lb.lbscan_gated_step(one, one, one, one[0], next(states), stream=s)],
        "norm": lambda s: values(lb.lbscan_norm_fwd(rows, w, w, residual=rows, return_stats=True, stream=s)),
        "norm gradients": lambda s: values(lb.lbscan_norm_bwd(None, w, dout=y, mean=mean, rstd=rstd, total=total, stream=s)),
        "embed": lambda s: [lb.lbscan_embed_fwd(ids, table, stream=s)],
        "embed gradient": lambda s: [lb.lbscan_embed_bwd(ids, dout=dout, vocab=5000, stream=s)],
    }


NAMES = ["gated", "gated again", "gated cut", "step", "norm", "norm gradients", "embed", "embed gradient"]


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
    sizes = [1 << k for k in range(9, 26)] + [v.numel() * v.element_size() for v in want]
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
    x = torch.randn(4, 16, device="cuda")
    s = torch.cuda.Stream()
    other = types.SimpleNamespace(cuda_stream=s.cuda_stream, stream_id=s.stream_id, device_index=s.device_index + 1,
                                  device_type=s.device_type)
    with pytest.raises(LbscanError, match="device") as e:
        lb.lbscan_norm_fwd(x, stream=other)
    assert e.value.code == EINVAL


def test_the_current_stream_named(lb):
    x = torch.randn(4, 16, device="cuda")
    assert torch.equal(lb.lbscan_norm_fwd(x, stream=torch.cuda.current_stream()), lb.lbscan_norm_fwd(x))

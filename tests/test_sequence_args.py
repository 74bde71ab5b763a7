"""What the operators around the scan refuse, on the host: struct layouts, sizes, pointers, tensors.  No GPU."""
import ctypes

import pytest
import torch

from paper_2506_15976_amd import binding, sequence
from paper_2506_15976_amd.autograd import gated_linear_recurrence, layer_norm, token_embedding
from paper_2506_15976_amd.binding import EINVAL, EUNSUPPORTED, EWORKSPACE, OK, LbscanError


@pytest.fixture(scope="module")
def lib():
    import os
    if not (os.path.exists(binding.LIB_PATH) and os.path.exists(sequence.TORCH_LIB_PATH)):
        from paper_2506_15976_amd import build
        build.build(force=True, verbose=False)
    return binding.load()


P = 4096                                          # an address that is never read


def gated(**k):
    a = binding.LbscanGatedArgs(2, 3, 64, 0, 0, 8.0, P, P, P, P, None, None, P, None, None, 0, None, 0)
    for name, v in k.items():
        setattr(a, name, v)
    return ctypes.byref(a)


def norm(**k):
    a = binding.LbscanNormArgs(5, 64, 0, 1e-5, P, None, P, P, P, None, P, P, None, 0)
    for name, v in k.items():
        setattr(a, name, v)
    return ctypes.byref(a)


def embed(**k):
    a = binding.LbscanEmbedArgs(5, 9, 64, 0, 1, 1.0, P, P, P, None, 0)
    for name, v in k.items():
        setattr(a, name, v)
    return ctypes.byref(a)


def test_struct_layouts():
    # 5 int32 and a float, 8 pointers, twice (pointer, size)
    assert ctypes.sizeof(binding.LbscanGatedArgs) == 24 + 8 * 8 + 2 * 16
    # int64, 2 int32, a float (padded), 8 pointers, (pointer, size)
    assert ctypes.sizeof(binding.LbscanNormArgs) == 24 + 8 * 8 + 16
    # int64, 4 int32, a float (padded), 3 pointers, (pointer, size)
    assert ctypes.sizeof(binding.LbscanEmbedArgs) == 32 + 3 * 8 + 16


@pytest.mark.parametrize("fields,code", [
    (dict(batch=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(seqlen=-1), EINVAL), (dict(dtype=2), EUNSUPPORTED),
    (dict(reverse=2), EINVAL), (dict(rate=float("nan")), EINVAL), (dict(rate=float("inf")), EINVAL),
    (dict(rate=-1.0), EINVAL), (dict(seqlen=(1 << 28) + 1), EUNSUPPORTED),
    (dict(batch=1 << 16, dim=1 << 16), EUNSUPPORTED), (dict(x=None), EINVAL), (dict(gate_a=None), EINVAL),
    (dict(gate_x=None), EINVAL), (dict(decay=None), EINVAL), (dict(y=None), EINVAL), (dict(x=P + 2), EINVAL),
    (dict(decay=P + 2), EINVAL), (dict(h0=P + 1), EINVAL), (dict(hT=P + 2), EINVAL), (dict(dtype=1, gate_a=P + 1), EINVAL),
    # rows that are cut, and no scratch for it
    (dict(batch=1, dim=1, seqlen=1 << 20), EWORKSPACE),
    (dict(batch=1, dim=1, seqlen=1 << 20, workspace=P, workspace_bytes=4), EWORKSPACE),
    # too little room for the states
    (dict(batch=1, dim=4096, seqlen=3000, saved_state=P, saved_state_bytes=4), EWORKSPACE),
])
def test_gated_forward_refuses(lib, fields, code):
    assert lib.lbscan_gated_fwd(gated(**fields), None) == code


def test_gated_backward_refuses(lib):
    grads = [P] * 7                               # dout dhT dx dgate_a dgate_x ddecay dh0
    assert lib.lbscan_gated_bwd(gated(), *grads, None) == EWORKSPACE
    for k in (0, 2, 3, 4, 5):
        g = list(grads)
        g[k] = None
        assert lib.lbscan_gated_bwd(gated(workspace=P, workspace_bytes=1 << 20), *g, None) == EINVAL
    g = list(grads)
    g[1] = P + 1
    assert lib.lbscan_gated_bwd(gated(workspace=P, workspace_bytes=1 << 20), *g, None) == EINVAL
    assert lib.lbscan_gated_bwd(gated(seqlen=3000, saved_state=P, saved_state_bytes=8), *grads, None) == EWORKSPACE
    assert lib.lbscan_gated_fwd(None, None) == EINVAL and lib.lbscan_gated_bwd(None, *grads, None) == EINVAL


@pytest.mark.parametrize("dtype", [0, 1])
def test_gated_scratch_follows_the_plan(lib, dtype):
    size = lambda which, **k: lib.lbscan_gated_workspace_bytes(gated(dtype=dtype, **k), which)  # noqa: E731
    FWD, BWD, SAVED = binding.WS_FWD, binding.WS_BWD, binding.WS_SAVED
    # a row in one tile: sums of q alone
    assert [size(w, seqlen=100) for w in (FWD, BWD, SAVED)] == [0, 6 * 4, 0]
    assert [size(w, seqlen=3) for w in (FWD, BWD, SAVED)] == [0, 6 * 4, 0]
    # several tiles: the states at their starts, kept by the caller or computed again
    many = dict(batch=64, dim=256, seqlen=60000)
    assert size(FWD, **many) == 0 and size(SAVED, **many) % (64 * 256 * 4) == 0 and size(SAVED, **many) > 0
    assert size(BWD, **many) == size(BWD, saved_state=P, **many) + size(SAVED, **many)
    # few long rows are cut
    assert size(FWD, batch=1, dim=2, seqlen=1 << 17) > 0
    assert size(FWD, seqlen=0) == 0 and size(99) == 0 and lib.lbscan_gated_workspace_bytes(None, FWD) == 0


@pytest.mark.parametrize("fields,code", [
    (dict(rows=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(dtype=5), EUNSUPPORTED), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(dim=(1 << 23) + 1), EUNSUPPORTED), (dict(rows=1 << 31), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(x=P + 2), EINVAL), (dict(weight=P + 2), EINVAL),
    (dict(residual=P), EINVAL), (dict(residual=P, sum=P + 1), EINVAL), (dict(mean=None), EINVAL), (dict(rstd=None), EINVAL),
    (dict(rows=0), OK), (dict(dim=0), OK),
])
def test_norm_forward_refuses(lib, fields, code):
    assert lib.lbscan_norm_fwd(norm(**fields), None) == code


def test_norm_backward_refuses(lib):
    room = dict(workspace=P, workspace_bytes=1 << 30)
    bwd = lambda args, dout=P, dsum=None, dx=P, dres=None, dw=P, db=P: lib.lbscan_norm_bwd(args, dout, dsum, dx, dres, dw, db, None)  # noqa: E731
    assert bwd(norm()) == EWORKSPACE
    assert bwd(norm(workspace=P, workspace_bytes=16)) == EWORKSPACE
    for bad in (dict(dout=None), dict(dx=None), dict(dsum=P), dict(dres=P), dict(dw=P + 1), dict(dout=P + 2)):
        assert bwd(norm(**room), **bad) == EINVAL, bad
    assert bwd(norm(mean=None, **room)) == EINVAL and bwd(norm(x=None, **room)) == EINVAL
    assert bwd(norm(residual=P, **room)) == EINVAL            # no sum
    assert bwd(None) == EINVAL


@pytest.mark.parametrize("fields,code", [
    (dict(tokens=-1), EINVAL), (dict(vocab=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(dtype=2), EUNSUPPORTED),
    (dict(ids_type=2), EUNSUPPORTED), (dict(scale=float("nan")), EINVAL), (dict(tokens=0x7fffffff), EUNSUPPORTED),
    (dict(dim=(1 << 23) + 1), EUNSUPPORTED), (dict(vocab=0), EINVAL), (dict(ids=None), EINVAL), (dict(ids=P + 4), EINVAL),
    (dict(ids_type=0, ids=P + 2), EINVAL), (dict(weight=None), EINVAL), (dict(out=P + 2), EINVAL), (dict(tokens=0), OK),
    (dict(dim=0), OK),
])
def test_embed_forward_refuses(lib, fields, code):
    assert lib.lbscan_embed_fwd(embed(**fields), None) == code


def test_embed_backward_refuses(lib):
    room = dict(workspace=P, workspace_bytes=1 << 30)
    assert lib.lbscan_embed_bwd(embed(), P, P, None) == EWORKSPACE
    assert lib.lbscan_embed_bwd(embed(**room), None, P, None) == EINVAL
    assert lib.lbscan_embed_bwd(embed(**room), P, None, None) == EINVAL
    assert lib.lbscan_embed_bwd(embed(ids=None, **room), P, P, None) == EINVAL
    assert lib.lbscan_embed_bwd(embed(vocab=0, **room), P, P, None) == EINVAL
    assert lib.lbscan_embed_bwd(None, P, P, None) == EINVAL
    assert lib.lbscan_embed_workspace_bytes(embed(tokens=1000)) > lib.lbscan_embed_workspace_bytes(embed()) > 0


# ---- the torch side: shapes and types are looked at before the device ------------------------------

def refused(code, f, *args, says="", **k):
    with pytest.raises(LbscanError) as e:
        f(*args, **k)
    assert e.value.code == code and says in str(e.value), str(e.value)


def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def test_tensors_not_on_the_device():
    row, decay = t(2, 3, 8), t(3)
    refused(EINVAL, sequence.lbscan_gated_fwd, row, row, row, decay, says="device tensor")
    refused(EINVAL, sequence.lbscan_gated_step, row[..., 0], row[..., 0], row[..., 0], decay, t(2, 3), says="device tensor")
    refused(EINVAL, sequence.lbscan_norm_fwd, row, says="device tensor")
    refused(EINVAL, sequence.lbscan_embed_fwd, t(4, dtype=torch.int64), t(5, 8), says="device tensor")
    refused(EINVAL, gated_linear_recurrence, row, row, row, decay, says="device tensor")
    refused(EINVAL, layer_norm, row, says="device tensor")
    refused(EINVAL, token_embedding, t(4, dtype=torch.int64), t(5, 8), says="device tensor")


def test_gated_binding_refuses():
    row = t(2, 3, 8)
    refused(EINVAL, sequence.lbscan_gated_fwd, t(2, 3), t(2, 3), t(2, 3), t(3), says="3 axes")
    half = t(2, 3, 8, dtype=torch.float16)
    refused(EUNSUPPORTED, sequence.lbscan_gated_fwd, half, half, half, t(3), says="dtype")
    refused(EINVAL, sequence.lbscan_gated_step, row, row, row, t(3), t(2, 3), says="2 axes")
    with pytest.raises(TypeError):
        sequence.lbscan_gated_step(row, row, row, t(3), None)


def test_norm_binding_refuses():
    x, m = t(4, 16), t(4)
    refused(EUNSUPPORTED, sequence.lbscan_norm_fwd, t(4, 16, dtype=torch.float16), says="dtype")
    refused(EINVAL, sequence.lbscan_norm_fwd, t(()), says="axis")
    refused(EINVAL, sequence.lbscan_norm_bwd, None, dout=x, mean=m, rstd=m, says="required")
    refused(EINVAL, sequence.lbscan_norm_bwd, x, dout=x, mean=m, rstd=m, dsum=x, says="dsum")


def test_embed_binding_refuses():
    ids = t(7, dtype=torch.int64)
    refused(EUNSUPPORTED, sequence.lbscan_embed_fwd, t(7), t(5, 8), says="int32 or int64")
    refused(EINVAL, sequence.lbscan_embed_fwd, ids, t(5, 8, 2), says="2 axes")
    refused(EINVAL, sequence.lbscan_embed_bwd, ids, dout=t(6, 8), vocab=5, says="shape of ids")
    refused(EINVAL, sequence.lbscan_embed_bwd, ids, dout=t(7), vocab=5, says="shape of ids")
    refused(EINVAL, sequence.lbscan_embed_bwd, ids, dout=t(7, 8), vocab=-1, says="vocab")

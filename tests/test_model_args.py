"""What the operators of state space language models refuse, on the host: struct layouts, sizes, pointers, tensors.  No GPU."""
import ctypes

import pytest
import torch

from paper_2506_15976_amd import binding, sequence
from paper_2506_15976_amd.autograd import block_norm, linear_cross_entropy
from paper_2506_15976_amd.binding import EINVAL, EUNSUPPORTED, EWORKSPACE, OK, LbscanError


@pytest.fixture(scope="module")
def lib():
    import os
    if not (os.path.exists(binding.LIB_PATH) and os.path.exists(sequence.TORCH_LIB_PATH)):
        from paper_2506_15976_amd import build
        build.build(force=True, verbose=False)
    return binding.load()


P = 4096                                          # an address that is never read


def filled(struct, given, fields):
    a = struct()
    for name, v in {**given, **fields}.items():
        setattr(a, name, v)
    return ctypes.byref(a)


def step(**k):
    names = ("x", "delta", "Bm", "Cm", "z", "A", "Dskip", "delta_bias", "conv_weight", "conv_bias", "conv_state", "state", "y")
    return filled(binding.LbscanStepArgs, dict(batch=2, dim=8, dstate=16, pool=2, conv_width=4, **dict.fromkeys(names, P)), k)


def prompt(**k):
    given = dict(batch=2, dim=8, seqlen=9, width=4, pool=2, x=P, weight=P, bias=P, state=P, y=P)
    return filled(binding.LbscanConvStateArgs, given, k)


def norm(**k):
    given = dict(rows=5, dim=64, norm_branch=1, norm_stream=1, eps=1e-5, residual_scale=1.0, x=P, gate=P, residual=P,
                 branch_weight=P, weight=P, y=P, sum=P, branch_rstd=P, stream_rstd=P)
    return filled(binding.LbscanBlockNormArgs, given, k)


def loss(**k):
    return filled(binding.LbscanLossArgs, dict(tokens=5, vocab=9, dim=64, ids_type=1, scale=1.0, x=P, weight=P, targets=P, loss=P, lse=P), k)


def test_struct_layouts():
    # int64, 4 int32, a float (padded), 5 pointers, (pointer, size)
    assert ctypes.sizeof(binding.LbscanLossArgs) == 32 + 5 * 8 + 16
    # 8 int32, 5 int64, 14 pointers
    assert ctypes.sizeof(binding.LbscanStepArgs) == 32 + 5 * 8 + 14 * 8
    # 7 int32 (padded), int64, 7 pointers
    assert ctypes.sizeof(binding.LbscanConvStateArgs) == 32 + 8 + 7 * 8
    # int64, 4 int32, 2 floats, 9 pointers, (pointer, size)
    assert ctypes.sizeof(binding.LbscanBlockNormArgs) == 32 + 9 * 8 + 16


@pytest.mark.parametrize("fields,code", [
    (dict(batch=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(dstate=-1), EINVAL), (dict(conv_width=-1), EINVAL),
    (dict(dtype=2), EUNSUPPORTED), (dict(delta_softplus=2), EINVAL), (dict(conv_activation=-1), EINVAL),
    (dict(conv_width=5), EUNSUPPORTED), (dict(dstate=17), EUNSUPPORTED), (dict(dstate=0), EUNSUPPORTED),
    (dict(batch=1 << 16, dim=1 << 16, pool=1 << 16), EUNSUPPORTED), (dict(batch=1, dim=(1 << 31) - 4095), EUNSUPPORTED), (dict(pool=1), EINVAL), (dict(pool=-1, slots=P), EINVAL),
    (dict(slots=P + 2), EINVAL), (dict(batch=65537, pool=70000, slots=P), EUNSUPPORTED),
    *[(dict([(name, None)]), EINVAL) for name in ("x", "delta", "Bm", "Cm", "A", "state", "y", "conv_weight", "conv_state")],
    *[(dict([(name, P + 2)]), EINVAL) for name in ("x", "z", "A", "Dskip", "delta_bias", "conv_weight", "conv_bias", "state", "y")],
    (dict(dtype=1, conv_state=P + 1), EINVAL), (dict(x_stride=7), EINVAL), (dict(delta_stride=-8), EINVAL), (dict(z_stride=1), EINVAL),
    (dict(b_stride=15), EINVAL), (dict(c_stride=1 << 40), EINVAL),
    (dict(batch=0), OK), (dict(dim=0), OK),
])
def test_step_refuses(lib, fields, code):
    assert lib.lbscan_step(step(**fields), None) == code


@pytest.mark.parametrize("fields,code", [
    (dict(batch=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(seqlen=-1), EINVAL), (dict(dtype=3), EUNSUPPORTED),
    (dict(width=0), EUNSUPPORTED), (dict(width=5), EUNSUPPORTED), (dict(activation=2), EINVAL),
    (dict(dim=1 << 16, seqlen=1 << 15), EUNSUPPORTED), (dict(dim=1, seqlen=(1 << 31) - 4095), EUNSUPPORTED),
    (dict(dim=1, seqlen=(1 << 31) - 1), EUNSUPPORTED), (dict(dim=(1 << 31) - 1, seqlen=1), EUNSUPPORTED), (dict(pool=1), EINVAL), (dict(pool=-3, slots=P), EINVAL),
    (dict(batch=65537, pool=70000, slots=P), EUNSUPPORTED),
    *[(dict([(name, None)]), EINVAL) for name in ("x", "weight", "state", "y")],
    *[(dict([(name, P + 2)]), EINVAL) for name in ("x", "weight", "bias", "state", "slots", "lengths", "y")],
    (dict(x_stride=71), EINVAL), (dict(batch=0), OK), (dict(dim=0), OK), (dict(seqlen=0), OK),
])
def test_prompt_refuses(lib, fields, code):
    assert lib.lbscan_conv1d_prompt(prompt(**fields), None) == code


@pytest.mark.parametrize("fields,code", [
    (dict(rows=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(dtype=5), EUNSUPPORTED), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(residual_scale=float("nan")), EINVAL),
    (dict(norm_branch=2), EINVAL), (dict(norm_stream=-1), EINVAL), (dict(norm_stream=0), EINVAL),
    (dict(dim=(1 << 23) + 1), EUNSUPPORTED), (dict(rows=1 << 31), EUNSUPPORTED), (dict(x=None), EINVAL), (dict(y=None), EINVAL),
    (dict(sum=None), EINVAL), *[(dict([(name, P + 2)]), EINVAL) for name in ("x", "gate", "residual", "branch_weight", "weight", "y",
                                                                          "sum", "branch_rstd", "stream_rstd")],
    (dict(rows=0), OK), (dict(dim=0), OK),
])
def test_norm_forward_refuses(lib, fields, code):
    assert lib.lbscan_block_norm_fwd(norm(**fields), None) == code


def test_norm_backward_refuses(lib):
    room = dict(workspace=P, workspace_bytes=1 << 30)

    def bwd(args, **k):
        given = dict(dout=P, dsum=P, dx=P, dgate=P, dresidual=P, dweight=P, dbranch=P)
        return lib.lbscan_block_norm_bwd(args, *{**given, **k}.values(), None)
    assert bwd(norm()) == EWORKSPACE and bwd(norm(workspace=P, workspace_bytes=16)) == EWORKSPACE
    for bad in (dict(dout=None), dict(dx=None), dict(dgate=None), dict(dout=P + 2), dict(dsum=P + 1), dict(dweight=P + 1),
                dict(dbranch=P + 2), dict(dresidual=P + 2)):
        assert bwd(norm(**room), **bad) == EINVAL, bad
    for bad in (dict(sum=None), dict(branch_rstd=None), dict(stream_rstd=None), dict(x=None), dict(residual=None), dict(gate=None),
                dict(norm_stream=0), dict(norm_stream=0, weight=None)):
        assert bwd(norm(**room, **bad)) == EINVAL, bad
    assert bwd(norm(rows=1 << 31, **room)) == EUNSUPPORTED and bwd(None) == EINVAL
    size = lib.lbscan_block_norm_workspace_bytes
    assert size(norm(rows=0)) == 0 and size(norm(dim=0)) == 0 and size(None) == 0
    # shares of both weights' gradients, one a block (of sixteen narrow rows), at most 512
    assert size(norm(rows=9)) == 2 * 64 * 4 and size(norm(rows=33)) == 3 * 2 * 64 * 4
    assert size(norm(rows=1 << 20, dim=1000)) == 512 * 2 * 1000 * 4
    # rows too long for registers: the rows' means, too
    assert size(norm(rows=1000, dim=20000)) == (256 * 2 * 20000 + 1000) * 4


@pytest.mark.parametrize("fields,code", [
    (dict(tokens=-1), EINVAL), (dict(vocab=-1), EINVAL), (dict(dim=-1), EINVAL), (dict(dtype=2), EUNSUPPORTED),
    (dict(ids_type=2), EUNSUPPORTED), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(tokens=(1 << 24) + 1), EUNSUPPORTED), (dict(vocab=1 << 30), EUNSUPPORTED), (dict(dim=0), EUNSUPPORTED),
    (dict(dim=65537), EUNSUPPORTED),
    *[(dict([(name, None)]), EINVAL) for name in ("x", "weight", "targets", "loss", "lse")],
    *[(dict([(name, P + 2)]), EINVAL) for name in ("x", "weight", "targets", "loss", "lse")], (dict(targets=P + 4), EINVAL),
    (dict(), EWORKSPACE), (dict(workspace=P, workspace_bytes=64), EWORKSPACE), (dict(workspace=P + 8, workspace_bytes=1 << 40), EWORKSPACE),
    (dict(tokens=0), OK),
])
def test_loss_forward_refuses(lib, fields, code):
    assert lib.lbscan_loss_fwd(loss(**fields), None) == code


def test_loss_backward_refuses(lib):
    room = dict(workspace=P, workspace_bytes=1 << 40)
    bwd = lambda args, dloss=P, dlse=P, dx=P, dw=P: lib.lbscan_loss_bwd(args, dloss, dlse, dx, dw, None)  # noqa: E731
    assert bwd(loss()) == EWORKSPACE and bwd(None) == EINVAL and bwd(loss(dim=0, **room)) == EUNSUPPORTED
    for bad in (dict(dloss=P + 2), dict(dlse=P + 1), dict(dx=P + 2), dict(dw=P + 1)):
        assert bwd(loss(**room), **bad) == EINVAL, bad
    assert bwd(loss(lse=None, **room)) == EINVAL and bwd(loss(), dx=None, dw=None) == OK
    size = lib.lbscan_loss_workspace_bytes
    assert size(loss(tokens=0), 0) == size(loss(vocab=0), 1) == size(loss(), 7) == size(None, 0) == size(loss(dim=0), 0) == 0
    # a table whose rows are no whole steps, or that is not aligned, has a copy
    big = dict(tokens=100, vocab=100000)
    assert size(loss(dim=64, **big), 0) + 100000 * 64 * 4 == size(loss(dim=64, weight=P + 4, **big), 0) == size(loss(dim=63, **big), 0)


def test_tensors_are_refused():
    """(meta and CPU tensors: no call gets as far as the GPU)"""
    cpu = lambda *s, **k: torch.zeros(*s, **k)  # noqa: E731
    x, A, B, state = cpu(2, 8), cpu(8, 4), cpu(2, 4), cpu(2, 8, 4)
    for call in (
        lambda: sequence.lbscan_step(x, x, A, B, B, state),
        lambda: sequence.lbscan_step(x.half(), x, A, B, B, state),
        lambda: sequence.lbscan_conv1d_step(x, cpu(2, 8, 3), cpu(8, 4)),
        lambda: sequence.lbscan_conv1d_prompt(cpu(2, 8, 5), cpu(2, 8, 3), cpu(8, 4)),
        lambda: sequence.lbscan_conv1d_prompt(cpu(2, 8, 5), cpu(2, 8, 4), cpu(8, 5)),
        lambda: sequence.lbscan_conv1d_prompt(cpu(2, 8), cpu(2, 8, 3), cpu(8, 4)),
        lambda: sequence.lbscan_block_norm_fwd(cpu(3, 5)),
        lambda: sequence.lbscan_block_norm_fwd(cpu(3, 5).double()),
        lambda: block_norm(cpu(3, 5)),
        lambda: sequence.lbscan_loss_fwd(cpu(3, 5), cpu(7, 5), cpu(3, dtype=torch.int64)),
        lambda: sequence.lbscan_loss_fwd(cpu(3, 5), cpu(7, 5), cpu(3)),
        lambda: sequence.lbscan_loss_fwd(cpu(3, 5).half(), cpu(7, 5).half(), cpu(3, dtype=torch.int64)),
        lambda: linear_cross_entropy(cpu(3, 5), cpu(7, 5), cpu(3, dtype=torch.int64)),
        lambda: sequence.lbscan_block_norm_bwd(cpu(3, 5), dout=cpu(3, 5)),
    ):
        with pytest.raises(LbscanError):
            call()


class TestOnTheDevice:
    """Shapes and types that do not fit, of device tensors."""
    pytestmark = pytest.mark.gpu

    @staticmethod
    def t(*shape, dtype=torch.float32):
        return torch.zeros(shape, device="cuda", dtype=dtype)

    @pytest.mark.parametrize("change", [
        dict(delta=(2, 9)), dict(Bm=(2, 5)), dict(A=(9, 4)), dict(state=(2, 8, 5)), dict(state=(3, 8, 4)), dict(z=(3, 8)),
        dict(conv_state=(2, 8, 2)), dict(conv_state=(1, 8, 3)), dict(conv_weight=(8, 5)), dict(conv_bias=(9,)), dict(slots=(3,)),
        dict(conv_state=None), dict(conv_weight=None), dict(Dskip=(9,)),
    ])
    def test_step(self, change):
        given = dict(x=(2, 8), delta=(2, 8), A=(8, 4), Bm=(2, 4), Cm=(2, 4), state=(2, 8, 4), conv_state=(2, 8, 3), conv_weight=(8, 4))
        t = {k: None if v is None else self.t(*v, dtype=torch.int32 if k == "slots" else torch.float32)
             for k, v in {**given, **change}.items()}
        with pytest.raises(LbscanError):
            sequence.lbscan_step(**t)

    def test_layouts_and_types(self):
        t = self.t
        x = t(2, 8)
        with pytest.raises(LbscanError):                     # columns that are not contiguous
            sequence.lbscan_step(t(2, 16)[:, ::2], x, t(8, 4), t(2, 4), t(2, 4), t(2, 8, 4))
        with pytest.raises(LbscanError):                     # rows that overlap
            sequence.lbscan_step(t(1, 8).expand(2, 8), x, t(8, 4), t(2, 4), t(2, 4), t(2, 8, 4))
        with pytest.raises(LbscanError):                     # a state that would have to be copied
            sequence.lbscan_step(x, x, t(8, 4), t(2, 4), t(2, 4), t(2, 4, 8).transpose(1, 2))
        with pytest.raises(LbscanError):
            sequence.lbscan_step(x, x, t(8, 4), t(2, 4), t(2, 4), t(2, 8, 4), slots=t(2, dtype=torch.int64))
        with pytest.raises(LbscanError):
            sequence.lbscan_step(x, x, t(8, 4), t(2, 4), t(2, 4), t(2, 8, 4), out=x)
        with pytest.raises(LbscanError):
            sequence.lbscan_conv1d_prompt(t(2, 8, 5), t(2, 8, 3), t(8, 4), lengths=t(2))
        with pytest.raises(LbscanError):
            sequence.lbscan_conv1d_prompt(t(2, 5, 8).transpose(1, 2), t(2, 8, 3), t(8, 4))
        y = t(3, 5)
        for call in (lambda: sequence.lbscan_block_norm_fwd(y, t(4)), lambda: sequence.lbscan_block_norm_fwd(y, t(5), norm_stream=False),
                     lambda: sequence.lbscan_block_norm_fwd(y, residual=t(3, 5, dtype=torch.bfloat16)),
                     lambda: sequence.lbscan_block_norm_fwd(y, out=y), lambda: sequence.lbscan_block_norm_fwd(y, gate=t(3, 6)),
                     lambda: sequence.lbscan_block_norm_bwd(y, dout=y), lambda: sequence.lbscan_block_norm_bwd(y, dout=y, stream_rstd=t(4)),
                     lambda: sequence.lbscan_block_norm_bwd(y, dout=y, stream_rstd=t(3), dsum=y),
                     lambda: sequence.lbscan_block_norm_fwd(t()),
                     lambda: sequence.lbscan_loss_fwd(y, t(7, 4), t(3, dtype=torch.int64)),
                     lambda: sequence.lbscan_loss_fwd(y, t(7, 5, dtype=torch.bfloat16), t(3, dtype=torch.int64)),
                     lambda: sequence.lbscan_loss_fwd(y, t(7, 5), t(4, dtype=torch.int64)),
                     lambda: sequence.lbscan_loss_fwd(y, t(7, 5), t(3, dtype=torch.int16)),
                     lambda: sequence.lbscan_loss_fwd(y, t(7, 10)[:, :5], t(3, dtype=torch.int64)),
                     lambda: sequence.lbscan_loss_fwd(t(3, 0), t(7, 0), t(3, dtype=torch.int64)),
                     lambda: sequence.lbscan_loss_bwd(y, t(7, 5), t(3, dtype=torch.int64), lse=t(4)),
                     lambda: sequence.lbscan_loss_bwd(y, t(7, 5), t(3, dtype=torch.int64), lse=t(3), dloss=t(3, dtype=torch.bfloat16))):
            with pytest.raises(LbscanError):
                call()

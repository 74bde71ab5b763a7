"""Operators of recurrent sequence models around the scan: gated linear recurrence, layer norm, token
embedding.  Argument marshalling only, like binding.py: every value is computed by the HIP kernels
behind include/lbscan.h, which defines what each call returns."""
from __future__ import annotations

import ctypes
import struct

from . import binding
from .binding import (EINVAL, EUNSUPPORTED, WS_BWD, WS_FWD, WS_SAVED, LbscanEmbedArgs, LbscanError, LbscanGatedArgs,
                      LbscanNormArgs, _address, _check, _dtype_code, _ptr, _stream, _tie_to_stream)


def _pack(layout, kind, *values):
    """A ctypes struct from its fields: one pack instead of an assignment per field."""
    try:
        return kind.from_buffer_copy(layout.pack(*values))
    except struct.error:
        raise LbscanError(EINVAL, f"sizes {values[:4]} do not fit the call") from None


def _expect(name, t, shape, dtype, optional=True):
    """Shape, type, device and layout of one tensor."""
    if t is None:
        if optional:
            return
        raise LbscanError(EINVAL, f"{name} is required")
    if t.shape != shape or t.dtype != dtype:
        raise LbscanError(EINVAL, f"{name}: expected {tuple(shape)} {dtype}, got {tuple(t.shape)} {t.dtype}")
    if not (t.is_cuda and t.is_contiguous()):
        raise LbscanError(EINVAL, f"{name} must be a contiguous device tensor")


def _scratch(nbytes, like, stream):
    """Scratch of one call (see binding._workspace_for), or None."""
    if not nbytes:
        return None
    import torch
    block = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    if stream is not None:
        block.record_stream(stream)
    return block


# ---- gated linear recurrence ---------------------------------------------------------------------

_GATED = struct.Struct("@5if8PPNPN")
assert _GATED.size == ctypes.sizeof(LbscanGatedArgs)
_MARKS = None


def _gated_args(x, gate_a, gate_x, decay, starts, h0, y, hT, rate, reverse, saved_state):
    import torch
    global _MARKS
    if _MARKS is None:
        _MARKS = (torch.bool, torch.uint8)
    B, D, L = x.shape
    code = _dtype_code(x)
    _expect("x", x, x.shape, x.dtype, False)
    _expect("gate_a", gate_a, x.shape, x.dtype, False)
    _expect("gate_x", gate_x, x.shape, x.dtype, False)
    _expect("decay", decay, (D,), torch.float32, False)
    if starts is not None:
        if starts.dtype not in _MARKS:
            raise LbscanError(EUNSUPPORTED, f"starts: expected bool or uint8, got {starts.dtype}")
        _expect("starts", starts, (B, L), starts.dtype)
    _expect("h0", h0, (B, D), torch.float32)
    _expect("hT", hT, (B, D), torch.float32)
    _expect("out", y, x.shape, x.dtype)
    if saved_state is not None:
        _expect("saved_state", saved_state, saved_state.shape, torch.float32)
    return _pack(_GATED, LbscanGatedArgs, B, D, L, code, int(bool(reverse)), float(rate), x.data_ptr(),
                 gate_a.data_ptr(), gate_x.data_ptr(), decay.data_ptr(), _address(starts), _address(h0), _address(y),
                 _address(hT), 0, 0, _address(saved_state), 0 if saved_state is None else saved_state.numel() * 4)


def _gated_scratch(args, which, like, stream):
    need = binding.load().lbscan_gated_workspace_bytes(ctypes.byref(args), which)
    ws = _scratch(need, like, stream)
    if ws is not None:
        args.workspace, args.workspace_bytes = ws.data_ptr(), need
    return ws


def lbscan_gated_saved_state(x, *, reverse=False):
    """Buffer for lbscan_gated_fwd(saved_state=...) / lbscan_gated_bwd(saved_state=...), or None when
    these sizes do not use one."""
    import torch
    B, D, L = x.shape
    a = _pack(_GATED, LbscanGatedArgs, B, D, L, _dtype_code(x), int(bool(reverse)), 0.0, *[0] * 12)
    need = binding.load().lbscan_gated_workspace_bytes(ctypes.byref(a), WS_SAVED)
    return torch.empty(need // 4, dtype=torch.float32, device=x.device) if need else None


def lbscan_gated_fwd(x, gate_a, gate_x, decay, *, rate=8.0, starts=None, reverse=False, h0=None,
                     return_state=False, out=None, saved_state=None, stream=None):
    """Gated linear recurrence along the last axis of x, gate_a, gate_x (B,D,L); decay (D) fp32.
    starts (B,L) bool or uint8: tokens at which a new sequence begins.  h0 (B,D) fp32: the state that enters;
    with return_state the result is (y, hT)."""
    import torch
    y = torch.empty_like(x) if out is None else out
    hT = torch.empty(x.shape[:2], dtype=torch.float32, device=x.device) if return_state else None
    a = _gated_args(x, gate_a, gate_x, decay, starts, h0, y, hT, rate, reverse, saved_state)
    ws = _gated_scratch(a, WS_FWD, x, stream)
    _tie_to_stream(stream, y if out is None else None, hT)
    _check(binding.load().lbscan_gated_fwd(ctypes.byref(a), _stream(stream)), "lbscan_gated_fwd")
    del ws
    return (y, hT) if return_state else y


def lbscan_gated_step(x, gate_a, gate_x, decay, state, *, rate=8.0, starts=None, out=None, stream=None):
    """One token of every sequence: x, gate_a, gate_x (B,D), state (B,D) fp32, which is updated in place;
    starts (B): sequences that begin with this token.  The result is the output (B,D)."""
    import torch
    if x.dim() != 2 or state is None:
        raise LbscanError(EINVAL, "a step takes x (B,D) and a state (B,D)")
    y = torch.empty_like(x) if out is None else out
    _expect("x", x, x.shape, x.dtype, False)
    _expect("gate_a", gate_a, x.shape, x.dtype, False)
    _expect("gate_x", gate_x, x.shape, x.dtype, False)
    _expect("decay", decay, x.shape[1:], torch.float32, False)
    _expect("state", state, x.shape, torch.float32, False)
    _expect("out", y, x.shape, x.dtype)
    if starts is not None:
        if starts.dtype not in (torch.bool, torch.uint8):
            raise LbscanError(EUNSUPPORTED, f"starts: expected bool or uint8, got {starts.dtype}")
        _expect("starts", starts, x.shape[:1], starts.dtype)
    B, D = x.shape
    s = state.data_ptr()
    a = _pack(_GATED, LbscanGatedArgs, B, D, 1, _dtype_code(x), 0, float(rate), x.data_ptr(), gate_a.data_ptr(),
              gate_x.data_ptr(), decay.data_ptr(), _address(starts), s, y.data_ptr(), s, 0, 0, 0, 0)
    _tie_to_stream(stream, y if out is None else None)
    _check(binding.load().lbscan_gated_fwd(ctypes.byref(a), _stream(stream)), "lbscan_gated_step")
    return y


def lbscan_gated_bwd(x, gate_a, gate_x, decay, *, dout, rate=8.0, starts=None, reverse=False, h0=None, dhT=None,
                     saved_state=None, stream=None):
    """Gradients of lbscan_gated_fwd: a dict with dx, dgate_a, dgate_x, ddecay and, with h0 or dhT (the
    gradient arriving at the state that leaves), dh0."""
    import torch
    a = _gated_args(x, gate_a, gate_x, decay, starts, h0, None, None, rate, reverse, saved_state)
    _expect("dout", dout, x.shape, x.dtype, False)
    _expect("dhT", dhT, x.shape[:2], torch.float32)
    g = dict(dx=torch.empty_like(x), dgate_a=torch.empty_like(x), dgate_x=torch.empty_like(x),
             ddecay=torch.empty_like(decay))
    if h0 is not None or dhT is not None:
        g["dh0"] = torch.empty(x.shape[:2], dtype=torch.float32, device=x.device)
    ws = _gated_scratch(a, WS_BWD, x, stream)
    _tie_to_stream(stream, *g.values())
    rc = binding.load().lbscan_gated_bwd(ctypes.byref(a), dout.data_ptr(), _ptr(dhT), g["dx"].data_ptr(),
                                         g["dgate_a"].data_ptr(), g["dgate_x"].data_ptr(), g["ddecay"].data_ptr(),
                                         _ptr(g.get("dh0")), _stream(stream))
    _check(rc, "lbscan_gated_bwd")
    del ws
    return g


# ---- layer norm ----------------------------------------------------------------------------------

_NORM = struct.Struct("@q2if8PPN")
assert _NORM.size == ctypes.sizeof(LbscanNormArgs)


def _norm_args(x, weight, bias, residual, y, total, mean, rstd, eps):
    import torch
    if x.dim() < 1:
        raise LbscanError(EINVAL, "x needs an axis to normalise")
    D = x.shape[-1]
    _expect("x", x, x.shape, x.dtype, False)
    _expect("weight", weight, (D,), torch.float32)
    _expect("bias", bias, (D,), torch.float32)
    _expect("residual", residual, x.shape, torch.float32)
    _expect("out", y, x.shape, x.dtype)
    _expect("sum", total, x.shape, torch.float32)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _expect(name, t, x.shape[:-1], torch.float32)
    return _pack(_NORM, LbscanNormArgs, x.numel() // D if D else 0, D, _dtype_code(x), float(eps), x.data_ptr(),
                 _address(residual), _address(weight), _address(bias), _address(y), _address(total), _address(mean),
                 _address(rstd), 0, 0)


def lbscan_norm_fwd(x, weight=None, bias=None, *, residual=None, eps=1e-5, return_stats=False, out=None,
                    stream=None):
    """Layer norm over the last axis of x; weight, bias (dim) fp32.  With residual (fp32, x's shape) the
    sum x + residual is normalised and the result is (y, sum), the sum in fp32; with return_stats the means
    and reciprocal deviations of the rows follow, for lbscan_norm_bwd."""
    import torch
    y = torch.empty_like(x) if out is None else out
    total = torch.empty_like(residual) if residual is not None else None
    mean = rstd = None
    if return_stats:
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
    a = _norm_args(x, weight, bias, residual, y, total, mean, rstd, eps)
    _tie_to_stream(stream, y if out is None else None, total, mean, rstd)
    _check(binding.load().lbscan_norm_fwd(ctypes.byref(a), _stream(stream)), "lbscan_norm_fwd")
    res = (y,) if total is None else (y, total)
    if return_stats:
        res += (mean, rstd)
    return res if len(res) > 1 else y


def lbscan_norm_bwd(x, weight=None, *, dout, mean, rstd, with_bias=True, total=None, dsum=None, stream=None):
    """Gradients of lbscan_norm_fwd: a dict with dx, dweight, dbias (None without weight / with_bias) and,
    where the forward call had a residual, dresidual (fp32).  total: the sum that the forward call returned (x is
    not read then and may be None); dsum: the gradient arriving at it."""
    import torch
    if mean is None or rstd is None or dout is None:
        raise LbscanError(EINVAL, "dout, and mean and rstd of the forward call, are required")
    if total is None and (x is None or dsum is not None):
        raise LbscanError(EINVAL, "x is required without a sum, and dsum belongs to one")
    if x is not None:
        _expect("x", x, dout.shape, dout.dtype)
    # (the type and the shape are dout's)
    a = _norm_args(dout, weight, None, total, None, total, mean, rstd, eps=0.0)
    a.x = _ptr(x)
    _expect("dsum", dsum, dout.shape, torch.float32)
    g = dict(dx=None, dresidual=None, dweight=None, dbias=None)
    if total is not None:
        g["dresidual"] = torch.empty_like(total)
    # in fp32 dx and dresidual are the same values
    shared = total is not None and dout.dtype == torch.float32
    g["dx"] = g["dresidual"] if shared else torch.empty_like(dout)
    D = dout.shape[-1]
    if weight is not None:
        g["dweight"] = torch.empty(D, dtype=torch.float32, device=dout.device)
    if with_bias:
        g["dbias"] = torch.empty(D, dtype=torch.float32, device=dout.device)
    need = binding.load().lbscan_norm_workspace_bytes(ctypes.byref(a))
    ws = _scratch(need, dout, stream)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _tie_to_stream(stream, *g.values())
    rc = binding.load().lbscan_norm_bwd(ctypes.byref(a), dout.data_ptr(), _ptr(dsum), None if shared else _ptr(g["dx"]),
                                        _ptr(g["dresidual"]), _ptr(g["dweight"]), _ptr(g["dbias"]), _stream(stream))
    _check(rc, "lbscan_norm_bwd")
    del ws
    return g


# ---- token embedding -------------------------------------------------------------------------------

_EMBED = struct.Struct("@q4if3PPN")
assert _EMBED.size == ctypes.sizeof(LbscanEmbedArgs)


def _ids_code(ids):
    import torch
    if ids.dtype == torch.int64:
        return 1
    if ids.dtype == torch.int32:
        return 0
    raise LbscanError(EUNSUPPORTED, f"ids: expected int32 or int64, got {ids.dtype}")


def _embed_args(ids, weight, vocab, dim, like, out, scale):
    _expect("ids", ids, ids.shape, ids.dtype, False)
    return _pack(_EMBED, LbscanEmbedArgs, ids.numel(), vocab, dim, _dtype_code(like), _ids_code(ids), float(scale),
                 ids.data_ptr(), _address(weight), _address(out), 0, 0)


def lbscan_embed_fwd(ids, weight, *, scale=1.0, out=None, stream=None):
    """scale * weight[ids]: ids int32 or int64 of any shape, weight (vocab, dim); zeros for ids that are no
    row of the table.  The result has the shape of ids and one more axis."""
    import torch
    _expect("weight", weight, weight.shape, weight.dtype, False)
    if weight.dim() != 2:
        raise LbscanError(EINVAL, f"weight: expected (vocab, dim), got {tuple(weight.shape)}")
    shape = ids.shape + weight.shape[1:]
    y = torch.empty(shape, dtype=weight.dtype, device=weight.device) if out is None else out
    _expect("out", y, shape, weight.dtype)
    a = _embed_args(ids, weight, weight.shape[0], weight.shape[1], weight, y, scale)
    _tie_to_stream(stream, y if out is None else None)
    _check(binding.load().lbscan_embed_fwd(ctypes.byref(a), _stream(stream)), "lbscan_embed_fwd")
    return y


def lbscan_embed_bwd(ids, *, dout, vocab, scale=1.0, stream=None):
    """Gradient of lbscan_embed_fwd with respect to the whole table, (vocab, dim) in dout's type: sums
    over the tokens of each row in fp32 and in the order of the tokens."""
    import torch
    _expect("dout", dout, ids.shape + dout.shape[-1:], dout.dtype, False)
    D = dout.shape[-1]
    dweight = torch.empty((int(vocab), D), dtype=dout.dtype, device=dout.device)
    a = _embed_args(ids, None, int(vocab), D, dout, None, scale)
    need = binding.load().lbscan_embed_workspace_bytes(ctypes.byref(a))
    ws = _scratch(need, dout, stream)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _tie_to_stream(stream, dweight)
    _check(binding.load().lbscan_embed_bwd(ctypes.byref(a), dout.data_ptr(), dweight.data_ptr(), _stream(stream)),
           "lbscan_embed_bwd")
    del ws
    return dweight

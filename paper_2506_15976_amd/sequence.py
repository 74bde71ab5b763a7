"""Operators of recurrent sequence models around the scan: gated linear recurrence, layer norm, token
embedding.  Names and defaults only: arguments are checked and the calls made in csrc/lbscan_torch.cpp, and every
value is computed by the HIP kernels behind include/lbscan.h, which defines what each call returns.
Refused arguments raise binding.LbscanError.

stream: a torch.cuda.Stream to run on instead of the current one.  The call does not wait for the current stream, so the
caller sees to it that the inputs (and tensors given to be written) are ready on that stream, and that the outputs
are before they are used on another.  Outputs and scratch are that stream's memory, and outputs are tied to the
current one.

out, and the state of a single step, are overwritten as in-place operations overwrite: autograd sees it by their versions, and
tensors that require gradients are refused while gradients are recorded."""
from __future__ import annotations

import importlib.util
import os

from . import binding

TORCH_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lbscan_torch.so")

_ext = None


def load():
    """The torch side of these operators (once); there is no fallback."""
    global _ext
    if _ext is None:
        binding.load()
        if not os.path.exists(TORCH_LIB_PATH):
            raise ImportError(f"{TORCH_LIB_PATH} is missing: build it with `python -m paper_2506_15976_amd.build`")
        spec = importlib.util.spec_from_file_location("_lbscan_torch", TORCH_LIB_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _ext = module
    return _ext


def lbscan_gated_saved_state(x, *, reverse=False, stream=None):
    """Buffer for lbscan_gated_fwd(saved_state=...) / lbscan_gated_bwd(saved_state=...), or None when
    these sizes do not use one.  stream: that of the calls it is for."""
    return (_ext or load()).gated_saved(x, reverse, stream)


def lbscan_gated_fwd(x, gate_a, gate_x, decay, *, rate=8.0, starts=None, reverse=False, h0=None,
                     return_state=False, out=None, saved_state=None, stream=None):
    """Gated linear recurrence along the last axis of x, gate_a, gate_x (B,D,L); decay (D) fp32.
    starts (B,L) bool or uint8: tokens at which a new sequence begins.  h0 (B,D) fp32: the state that enters;
    with return_state the result is (y, hT)."""
    return (_ext or load()).gated_fwd(x, gate_a, gate_x, decay, starts, h0, rate, reverse, return_state, out,
                                      saved_state, stream)


def lbscan_gated_step(x, gate_a, gate_x, decay, state, *, rate=8.0, starts=None, out=None, stream=None):
    """One token of every sequence: x, gate_a, gate_x (B,D), state (B,D) fp32, which is updated in place;
    starts (B): sequences that begin with this token.  The result is the output (B,D)."""
    return (_ext or load()).gated_step(x, gate_a, gate_x, decay, state, starts, rate, out, stream)


def lbscan_gated_bwd(x, gate_a, gate_x, decay, *, dout, rate=8.0, starts=None, reverse=False, h0=None, dhT=None,
                     saved_state=None, stream=None):
    """Gradients of lbscan_gated_fwd: a dict with dx, dgate_a, dgate_x, ddecay and, with h0 or dhT (the
    gradient arriving at the state that leaves), dh0."""
    return (_ext or load()).gated_bwd(x, gate_a, gate_x, decay, dout, starts, h0, dhT, rate, reverse, saved_state, stream)


def lbscan_norm_fwd(x, weight=None, bias=None, *, residual=None, eps=1e-5, return_stats=False, out=None,
                    stream=None):
    """Layer norm over the last axis of x; weight, bias (dim) fp32.  With residual (fp32, x's shape) the
    sum x + residual is normalised and the result is (y, sum), the sum in fp32; with return_stats the means
    and reciprocal deviations of the rows follow, for lbscan_norm_bwd (zeros where rows have no columns)."""
    return (_ext or load()).norm_fwd(x, weight, bias, residual, eps, return_stats, out, stream)


def lbscan_norm_bwd(x, weight=None, *, dout, mean, rstd, with_bias=True, total=None, dsum=None, stream=None):
    """Gradients of lbscan_norm_fwd: a dict with dx, dweight, dbias (None without weight / with_bias) and,
    where the forward call had a residual, dresidual (fp32).  total: the sum that the forward call returned (x is
    not read then and may be None); dsum: the gradient arriving at it."""
    return (_ext or load()).norm_bwd(x, weight, dout, mean, rstd, with_bias, total, dsum, stream)


def lbscan_embed_fwd(ids, weight, *, scale=1.0, out=None, stream=None):
    """scale * weight[ids]: ids int32 or int64 of any shape, weight (vocab, dim); zeros for ids that are no
    row of the table.  The result has the shape of ids and one more axis."""
    return (_ext or load()).embed_fwd(ids, weight, scale, out, stream)


def lbscan_embed_bwd(ids, *, dout, vocab, scale=1.0, stream=None):
    """Gradient of lbscan_embed_fwd with respect to the whole table, (vocab, dim) in dout's type: sums
    over the tokens of each row in fp32 and in the order of the tokens."""
    return (_ext or load()).embed_bwd(ids, dout, vocab, scale, stream)

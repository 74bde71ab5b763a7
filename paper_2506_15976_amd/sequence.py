"""Operators of recurrent and state space sequence models around the scan: gated linear recurrence, layer norm, token
embedding; the scan's and the convolution's forms for serving, the norms around a block, the loss over a vocabulary.  Names and defaults
only: arguments are checked and the calls made in csrc/lbscan_torch*.cpp, and every
value is computed by the HIP kernels behind include/lbscan.h, which defines what each call returns.
Refused arguments raise binding.LbscanError.

stream: a torch.cuda.Stream to run on instead of the current one.  The call does not wait for the current stream, so the
caller sees to it that the inputs (and tensors given to be written) are ready on that stream, and that the outputs
are before they are used on another.  Outputs and scratch are that stream's memory, and outputs are tied to the
current one.

out, and the states of steps and prompts, are overwritten as in-place operations overwrite: autograd sees it by their versions, and
tensors that require gradients are refused while gradients are recorded.  Of steps and prompts of the scan and its convolution, and of
the norms around a block, they share no memory with what the call reads or writes besides (refused)."""
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


def lbscan_step(x, delta, A, Bm, Cm, state, Dskip=None, z=None, delta_bias=None, *, delta_softplus=True, conv_state=None,
                conv_weight=None, conv_bias=None, activation=True, slots=None, out=None, stream=None):
    """One token of every sequence through the selective scan: x, delta, z (B,D), Bm, Cm (B,N), which may be columns of
    wider tensors, A (D,N), state (B,D,N) fp32, which is updated in place.  With conv_weight (D,K) x goes through the
    convolution (and SiLU, unless activation is off) first, whose last K-1 inputs are conv_state (B,D,K-1) in x's type, updated in
    place too.  slots (B) int32: rows of larger states, (S,D,N) and (S,D,K-1), that belong to the rows of x; a row whose slot
    is none of them, or an earlier row's, is padding: its output is zero and no state is touched for it.  The
    result is the output (B,D)."""
    return (_ext or load()).step(x, delta, A, Bm, Cm, state, Dskip, z, delta_bias, delta_softplus, conv_state, conv_weight,
                                 conv_bias, activation, slots, out, stream)


def lbscan_conv1d_step(x, state, weight, bias=None, *, activation=True, slots=None, out=None, stream=None):
    """One token of every sequence through the convolution: x (B,D), which may be columns of a wider tensor; state and
    slots as conv_state and slots of lbscan_step."""
    return (_ext or load()).conv1d_prompt(x, state, weight, bias, activation, None, slots, out, True, stream)


def lbscan_conv1d_prompt(x, state, weight, bias=None, *, activation=True, lengths=None, slots=None, out=None, stream=None):
    """Prompts, or pieces of them, through the convolution: x (B,D,L); the K-1 tokens before them are those of state
    (zeros before a sequence), which leaves with the last K-1 inputs.  lengths (B) int32: tokens of each row that are there; the
    output is zero behind them.  state and slots as conv_state and slots of lbscan_step."""
    return (_ext or load()).conv1d_prompt(x, state, weight, bias, activation, lengths, slots, out, False, stream)


def lbscan_block_norm_fwd(x, weight=None, *, gate=None, branch_weight=None, residual=None, residual_scale=1.0,
                          norm_branch=False, norm_stream=True, eps=1e-5, return_stats=False, out=None, stream=None):
    """The norms (root mean square) around a block over the last axis of x, its output: x SiLU(gate), normalised with
    norm_branch, times branch_weight, is added to residual_scale * residual (fp32), and the sum, normalised with norm_stream
    and times weight, is returned; with a residual (y, sum), the sum in fp32.  branch_weight, weight (dim) fp32.  With
    return_stats the reciprocal deviations of the branch and of the stream follow (None without the norm)."""
    return (_ext or load()).block_norm_fwd(x, weight, gate, branch_weight, residual, residual_scale, norm_branch, norm_stream,
                                           eps, return_stats, out, stream)


def lbscan_block_norm_bwd(x, weight=None, *, dout, gate=None, branch_weight=None, total=None, dsum=None, branch_rstd=None,
                          stream_rstd=None, residual_scale=1.0, norm_branch=False, norm_stream=True, stream=None):
    """Gradients of lbscan_block_norm_fwd: a dict with dx, dgate, dresidual (fp32), dweight, dbranch_weight, None for what the
    forward call did not have.  total: the sum that it returned; dsum: the gradient arriving at it; branch_rstd,
    stream_rstd: its statistics."""
    return (_ext or load()).block_norm_bwd(x, weight, dout, gate, branch_weight, total, dsum, branch_rstd, stream_rstd,
                                           residual_scale, norm_branch, norm_stream, stream)


def lbscan_loss_fwd(x, weight, targets, *, scale=1.0, stream=None):
    """Softmax cross entropy of tokens over a vocabulary: x (..., dim), weight (vocab, dim) in one type, targets (...) int32 or
    int64.  The logits scale * x weight^T are never kept.  The result is (loss, lse), fp32 in the shape of targets; zeros for
    tokens whose target is no row of the table, which are left out."""
    return (_ext or load()).loss_fwd(x, weight, targets, scale, stream)


def lbscan_loss_bwd(x, weight, targets, *, lse, dloss=None, dlse=None, scale=1.0, stream=None):
    """Gradients of lbscan_loss_fwd: a dict with dx and dweight, in x's type; lse as it was returned; dloss, dlse fp32: the
    gradients of loss and lse (None: zeros)."""
    return (_ext or load()).loss_bwd(x, weight, targets, lse, dloss, dlse, scale, stream)

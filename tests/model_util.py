"""Tolerances and helpers for the GPU tests of the operators of state space language models.

Errors are those of sequence_util.close: max |got - ref| / max(|ref|, 0.1 rms(ref)) and mean |got - ref| / rms(ref).
With u = 2^-24:

 * step: dt by softplus (4 u), exp2 and its argument (a factor x e^-x (3 u) <= 1.1 u, and 2 u), three products: a state is off
   by at most 12 u of |a h| + |dt B x|.  y adds 17 terms of which each carries that and the sum's 17 u: 30 u of the sum of
   their sizes, which is about 4 rms; at the floor's tenth 30 u * 4 * 10 = 7e-5, to 1e-4.  Mean: 30 u = 2e-6, to 5e-6.
 * convolution: 4 products and sums, SiLU (6 u): 10 u of the sum of sizes, 2 rms; at the floor's tenth 10 u * 2 * 10 = 1.2e-5,
   and where SiLU bends down its slope is at most 1.1: to 5e-5.  Mean 1e-6.
 * norms: the layer norm's 80 u = 5e-6 for each of two norms, gate 6 u more, at the floor's tenth: to 4e-5, mean 2e-6.
   Gradients: two times three terms that cancel, about 25 roundings: 25 u * 10 * 3 = 4.5e-5, to 1e-4, mean 5e-6.  They are
   differences h - hat mean(h hat) times a factor, each term rounded by itself: the error goes by the size of the terms (h alone,
   the gradient with the deviations held), not by that of the difference, which for a row of one column is h (1 - hat^2), about
   eps of h.  So rms is that of the larger of the two (close_terms).
 * bf16 outputs: the result is rounded once, by at most 2^-8 of it (half a step), on top of that of fp32; the mean of the
   roundings, too, is at most 2^-8 of the mean of |ref|, which is at most rms(ref) (both are reached by a single value).
"""
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = 2.0 ** -8


def tolerances(fp32):
    return {torch.float32: fp32, torch.bfloat16: (HALF_STEP + fp32[0], HALF_STEP + fp32[1])}


STEP = tolerances((1e-4, 5e-6))
CONV = tolerances((5e-5, 1e-6))
NORM = tolerances((4e-5, 2e-6))
NORM_GRADIENT = tolerances((1e-4, 5e-6))


def close_terms(got, want, terms, tol, what):
    """As sequence_util.close, with the size of the terms whose difference `want` is."""
    got = got.detach().double().cpu()
    size = max(float(want.square().mean().sqrt()), float(terms.square().mean().sqrt()))
    error = (got - want).abs()
    worst, mean = float((error / want.abs().clamp(min=max(0.1 * size, 1e-300))).max()), float(error.mean()) / (size or 1.0)
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    assert worst <= tol[0] and mean <= tol[1], f"{what}: error {worst:.2e} (<= {tol[0]}), mean {mean:.2e} (<= {tol[1]})"


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def guarded(t, beyond=64):
    """The same values with a margin of a known pattern on both sides, and a function that says whether it still stands."""
    margin = torch.arange(beyond, device=t.device).to(t.dtype)
    flat = torch.cat([margin, t.reshape(-1), margin])
    inner = flat[beyond:beyond + t.numel()].view(t.shape)
    return inner, lambda: bool((flat[:beyond] == margin).all() and (flat[beyond + t.numel():] == margin).all())

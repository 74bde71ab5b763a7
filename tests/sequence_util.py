"""Helpers for the GPU tests of the operators around the scan.

Tolerances, of the scale-aware error max |got - ref| / max(|ref|, 0.1 rms(ref)) and of mean |got - ref| / rms(ref),
as multiples of the rounding unit u = 2^-24 (fp32) and 2^-9 (bf16 outputs, one rounding of a result in fp32):

 * recurrence, fp32: a token's a is off by at most about 8 u (exp2, its argument, the logistic function), and the
   state remembers up to 1 / (1 - a) ~ 2000 tokens with independent errors: 8 u sqrt(2000) = 2e-5 of a state, five
   times that at the floor's tenth and over millions of outputs: 1e-4.  Mean over channels, memories of
   about 100 tokens: 8 u sqrt(100) = 5e-6.
 * norm, fp32: about eight roundings, ten times that at the floor's tenth: 80 u = 5e-6, sums of 10^4 values
   in parts of a few tens each add as much again: 2e-5.  Mean: 8 u = 5e-7; column sums: 1e-6.
 * bf16: u / 2 of each output; at the floor's tenth ten times that: 1e-2 ... 2e-2, mean 4e-3.
"""
import numpy as np
import torch

from paper_2506_15976_amd.inputs import error_metric, mean_error

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
GATED = {"fp32": (1e-4, 5e-6), "bf16": (2e-2, 4e-3)}
NORM = {"fp32": (2e-5, 1e-6), "bf16": (2e-2, 4e-3)}


def to_numpy(t):
    return t.detach().double().cpu().numpy()


def close(got, want, tol, what):
    got = to_numpy(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, f"{what}: {got.shape}, expected {want.shape}"
    if not want.size:
        return
    assert np.all(np.isfinite(got)), f"{what}: non-finite values"
    if not np.any(want):
        assert not np.any(got), what
        return
    err, mean = error_metric(got, want), mean_error(got, want)
    assert err <= tol[0] and mean <= tol[1], f"{what}: error {err:.2e} (<= {tol[0]}), mean {mean:.2e} (<= {tol[1]})"


def off_by_one(t):
    """The same values in memory that starts one element behind an aligned address."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:]
    flat.copy_(t.reshape(-1))
    return flat.view(t.shape)

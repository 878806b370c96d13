"""What the tests of the recurrence, the linear layers and the 8-bit activations share.

Tolerances.  A result is rounded once to its type: half a step.  Before that:

  the recurrence: steps of 2^-24 relative to the terms that make a value up (oracle/layers_oracle.py sums their magnitudes along the
  recurrence).  fp32: a sigmoid is off by 7 steps (exponential and its correction 4, sum 1, reciprocal 2), the exponent rate * s by 8, a
  by 8 * exponent + 4, m^2 by 21 (series or difference), m by 14, the new value m i x by 14 + 7 + 2 = 23: 24 cover each.  16-bit types,
  gates within +-6: the exponential's argument is rounded, a sigmoid is off by 1.5 * 6 + 5 = 14, the exponent by 15, a by 16.5 *
  exponent + 2, m^2 by 53 (32 of them the series'), m by 30, the new value by 46: 48.  Gradients chain two such values and a product or
  two: twice as many and 8.
  sums of n terms: n steps of the sum of the terms' magnitudes."""
import numpy as np
import torch

from tests.block_parity import TORCH, f64, half_step, stored  # noqa: F401

STEPS = {"f32": 24, "f16": 48, "bf16": 48}
CODE = {"f32": 0, "f16": 1, "bf16": 2}


def within(got, ref, tol, what):
    got, ref = f64(got) if isinstance(got, torch.Tensor) else got, np.asarray(ref)
    assert got.shape == ref.shape, f"{what}: {got.shape} and {ref.shape}"
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    if not ref.size:
        return
    tol = np.broadcast_to(tol, ref.shape)
    over = np.abs(got - ref) - tol
    worst = np.unravel_index(np.argmax(over), over.shape)
    assert over.max() <= 0, f"{what}: {got[worst]!r} where {ref[worst]!r} is right (at {worst}; allowed {tol[worst]:.3e})"


def near(got, ref, dtype, steps, scale, what):
    within(got, ref, half_step(ref, dtype) + steps * 2.0 ** -24 * scale, what)


def live(shape, lengths):
    """Which tokens of [B, N, ...] count."""
    n = np.arange(shape[1])[None]
    return n < (np.full(shape[0], shape[1]) if lengths is None else np.clip(lengths, 0, shape[1]))[:, None]


def columns(parts, pad=0):
    """The tensors side by side as columns of one [B, N, sum] GPU buffer with `pad` values between them; returns the views."""
    B, N = parts[0].shape[:2]
    wide = sum(p.shape[2] + pad for p in parts)
    flat = torch.full((B, N, wide), float("nan"), dtype=parts[0].dtype, device="cuda")
    views, at = [], 0
    for p in parts:
        v = flat[..., at:at + p.shape[2]]
        v.copy_(p)
        views.append(v)
        at += p.shape[2] + pad
    return views

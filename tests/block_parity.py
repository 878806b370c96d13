"""Tolerance rule of the operators around the mixer (shared by their GPU tests).

A result is rounded once to its type: half a step, eps / 2 relative to the value (half the spacing of the subnormals below
the smallest normal).  Before that the arithmetic is fp32 (or sums of bf16 terms that carry 24 bits): an inner product of n
terms is off by at most n 2^-24 of the sum of its terms' magnitudes, to first order, and a result that is a chain of such
products by the sum of their n.  So

    |got - ref| <= half_step(ref) + n 2^-24 scale

with `n` the length of the chain and `scale` the largest magnitude the sums reach (the largest result where nothing says
more; for gradients that cancel, the sum of their terms)."""
import numpy as np
import torch

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(ref, dtype):
    info = torch.finfo(TORCH[dtype])
    return np.maximum(np.abs(ref) * info.eps / 2, info.smallest_normal * info.eps / 2)


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def check(got, ref, dtype, n, what, scale=None):
    got, ref = f64(got), np.asarray(ref)
    assert got.shape == ref.shape, f"{what}: {got.shape} and {ref.shape}"
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    if not ref.size:
        return 0.0
    scale = np.abs(ref).max() if scale is None else scale
    over = np.abs(got - ref) - half_step(ref, dtype) - n * 2.0 ** -24 * scale
    worst = np.unravel_index(np.argmax(over), over.shape)
    assert over.max() <= 0, (f"{what}: {got[worst]!r} where {ref[worst]!r} is right (at {worst}; allowed "
                             f"{(half_step(ref, dtype) + n * 2.0 ** -24 * scale)[worst]:.3e})")
    return float(np.abs(got - ref).max())


def stored(x, dtype):
    """fp64 numpy values as a CPU tensor of the type, and the values it holds."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[dtype])
    return t, t.to(torch.float64).numpy()

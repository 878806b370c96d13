"""GELU and its slope of 16-bit types where they are small: relative to themselves, as far out as the exponential is a normal fp32 number.

The tail Q of the normal distribution is off by 1.7e-5 of itself by its polynomial.  Its exponential's argument is rounded three times (the
square, the constant, their product): 3 z^2 / 2 steps of 2^-24; the reciprocal, six multiply-adds and two products are 16 steps at most.  The
slope adds z times the density, with the same exponential."""
import math

import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from tests.layers_parity import CODE, TORCH, half_step, within

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [60, 3000])   # few tokens; tiles
def test_gelu_of_values_far_below_zero(rows, dtype):
    z = -torch.linspace(0.0, 13.0, rows, dtype=torch.float64).to(TORCH[dtype])
    x = torch.zeros((1, rows, 8), dtype=TORCH[dtype])
    x[0, :, 0] = z
    w = torch.eye(8, dtype=TORCH[dtype], device="cuda")
    y, dx, dy = (torch.empty((1, rows, 8), dtype=TORCH[dtype], device="cuda") for _ in range(3))
    dy.fill_(1.0)
    n = max(lf.linfusion_linear_workspace_bytes(1, rows, 8, 8, CODE[dtype]), lf.linfusion_linear_bwd_workspace_bytes(1, rows, 8, 8, CODE[dtype]))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    lf.linfusion_linear_fwd(x.cuda(), w, None, y, activation=lf.ACT_GELU, workspace=ws)
    lf.linfusion_linear_bwd(None, w, x.cuda(), dy, dx=dx, activation=lf.ACT_GELU, workspace=ws)
    v = z.double().numpy()
    q = np.array([0.5 * math.erfc(-t / math.sqrt(2.0)) for t in v])
    density = np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    steps = (1.5 * v * v + 16) * U
    ref = v * q
    within(y[0, :, 0], ref, half_step(ref, dtype) + (1.7e-5 + steps) * np.abs(ref), "gelu")
    ref = q + v * density
    within(dx[0, :, 0], ref, half_step(ref, dtype) + (1.7e-5 + steps) * q + (steps + 4 * U) * np.abs(v) * density, "slope")

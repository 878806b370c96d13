"""Every tile shape of the linear layers' products, with k in one piece and in three, against fp64: tokens that one stride leads through, batch
rows of ragged lengths (of many tokens, and of a few), each size with a rest in every tile.  The choice by cost takes most of these shapes at sizes
only that are too large for an oracle."""
import numpy as np
import pytest

from tests.test_gpu_linear import backward, check_backward, check_forward, forward, make, on_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("tuning")]

LAYOUTS = {"flat": (1, 600, None), "rows": (4, 200, (200, 0, 77, 129)), "few a row": (40, 15, tuple((7 * b + 3) % 16 for b in range(40)))}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("dtype,shape", [(d, s) for d in ("bf16", "f16", "f32") for s in range(1, 9) if d != "f32" or s > 1], ids=str)
def test_every_shape(dtype, shape, splits, layout, monkeypatch):
    monkeypatch.setenv("LINFUSION_LINEAR_TILES", str(shape))
    monkeypatch.setenv("LINFUSION_LINEAR_SPLITS", str(splits))
    B, N, lengths = LAYOUTS[layout]
    c = make(B, N, 328, 520, dtype, shape, "silu", True, True, lengths)
    g = on_gpu(c)
    y, z = forward(c, g)
    check_forward(c, y, z)
    check_backward(c, backward(c, g))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["none", "leaky"])
def test_gradients_that_the_type_holds_are_not_rounded_before_the_products(act, dtype):
    """Without an activation, and with a slope of a half, dz is a value of the type: the results are rounded once."""
    import paper_2409_02097_amd as lf
    import torch
    from oracle import layers_oracle as orc
    from tests.layers_parity import CODE, f64, half_step, within
    B, N, K, C = 1, 700, 328, 520
    c = make(B, N, K, C, dtype, 3, act)
    g, w = on_gpu(c), c["w"]
    d = {n: torch.empty(s, dtype=g["dy"].dtype, device="cuda") for n, s in (("dx", (B, N, K)), ("dw", (C, K)), ("dbias", (C,)))}
    lf.linfusion_linear_bwd(g["x"], g["w"], g["z"] if act != "none" else None, g["dy"], **d, slope=0.5,
                            activation=lf.ACT_LEAKY_RELU if act == "leaky" else lf.ACT_NONE,
                            workspace=torch.empty(lf.linfusion_linear_bwd_workspace_bytes(B, N, K, C, CODE[dtype]), dtype=torch.uint8, device="cuda"))
    dz = (w["dy"] * orc.act(w["z"], act, 0.5)[1])[0]
    for n, ref, mag, terms in (("dx", dz @ w["w"], np.abs(dz) @ np.abs(w["w"]), C), ("dw", dz.T @ w["x"][0], np.abs(dz).T @ np.abs(w["x"][0]), N),
                               ("dbias", dz.sum(0), np.abs(dz).sum(0), N)):
        within(f64(d[n]).reshape(ref.shape), ref, half_step(ref, dtype) + (terms + 4) * 2.0 ** -24 * mag, n)

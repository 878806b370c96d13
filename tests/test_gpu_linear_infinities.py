"""Gradients of linear layers of 16-bit types where something is infinite or no number."""
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import layers_oracle as orc
from tests.layers_parity import CODE
from tests.test_gpu_linear import backward, make, memory, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lengths", [None, (700,)], ids=["flat", "rows"])
def test_infinities_stay_infinities(lengths, dtype):
    """What one factor makes infinite is infinite, of the sign of the other one, and no NaN; a NaN is one; other channels do not see them."""
    c = make(1, 700, 72, 136, dtype, 3, "silu", lengths=lengths)
    g = on_gpu(c)
    clean = backward(c, g)
    dz = torch.from_numpy(c["w"]["dy"] * orc.act(c["w"]["z"], "silu")[1]).cuda()[0]
    x, w = g["x"], g["w"]
    x[0, 5, 3], x[0, 400, 9], x[0, 650, 70], w[7, 2], w[100, 11], w[135, 71] = (float(v) for v in ("inf", "-inf", "nan", "-inf", "inf", "nan"))
    d = backward(c, g)
    inf = float("inf")
    assert torch.equal(d["dw"][:, 3].double(), torch.sign(dz[5]) * inf) and torch.equal(d["dw"][:, 9].double(), torch.sign(dz[400]) * -inf)
    assert torch.equal(d["dx"][0, :, 2].double(), torch.sign(dz[:, 7]) * -inf) and torch.equal(d["dx"][0, :, 11].double(), torch.sign(dz[:, 100]) * inf)
    assert bool(torch.isnan(d["dw"][:, 70]).all()) and bool(torch.isnan(d["dx"][0, :, 71]).all())
    for n, out, at in (("dw", d["dw"], (3, 9, 70)), ("dx", d["dx"][0], (2, 11, 71))):
        rest = [i for i in range(72) if i not in at]
        assert torch.equal(out[:, rest], clean[n].reshape(out.shape)[:, rest]), n


def test_an_infinite_gradient_is_one_where_the_type_ends():
    """dz beyond fp16's largest value is infinite, as rounded; so are the products with what is not 0."""
    n = 100
    dy = torch.full((1, n, 8), 65504.0, dtype=torch.float16, device="cuda")
    z = torch.full((1, n, 8), 2.4, dtype=torch.float16, device="cuda")   # silu's slope is 1.0998 there
    w = torch.ones((8, 8), dtype=torch.float16, device="cuda")
    dx, dw = torch.empty_like(dy), torch.empty_like(w)
    lf.linfusion_linear_bwd(dy, w, z, dy, dx=dx, dw=dw, activation=lf.ACT_SILU, workspace=memory(lf.linfusion_linear_bwd_workspace_bytes(1, n, 8, 8, CODE["f16"])))
    assert bool((dx == float("inf")).all()) and bool((dw == float("inf")).all())

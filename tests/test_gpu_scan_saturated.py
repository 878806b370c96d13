"""Gradients of gates of the recurrence that are nearly open or shut: the slope of a sigmoid, s (1 - s), where s no longer holds 1 - s.

As in layers_parity, with arguments up to 20 (fp32: 40) in place of 6.  fp32 adds what an argument's rounding loses, so its steps stay.  16-bit types: a sigmoid is
off by 1.5 * 20 + 5 = 35 steps, the exponent by 36, m by 40, the new value by 77: 80.  Relative to the slope: both factors of s (1 - s) are as
exact as the sigmoid that is the smaller one."""
import numpy as np
import pytest

from oracle import layers_oracle as orc
from tests.layers_parity import f64, near, stored
from tests.test_gpu_scan import backward, forward, make, on_gpu, reference

pytestmark = pytest.mark.gpu

STEPS = {"f32": 24, "f16": 80, "bf16": 80}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight,inputs,reverse", [("norm", True, False), ("norm", False, True), ("leaky", True, False), ("sum", True, True)])
@pytest.mark.parametrize("B,N,C", [(2, 300, 64), (1, 100, 40), (9, 5, 72)])   # several chunks, one, rows that share a workgroup
def test_slopes_of_saturated_gates(B, N, C, weight, inputs, reverse, dtype):
    c = make(B, N, C, dtype, N + C, weight, inputs, True, reverse)
    far, r = 40.0 if dtype == "f32" else 20.0, np.random.RandomState(4)
    for n in ("gate", "input") if inputs else ("gate",):
        c["t"][n], c["w"][n] = stored(r.uniform(-far, far, (B, N, C)), dtype)
    g = on_gpu(c)
    d = backward(c, g, forward(c, g)[2])
    w, held = c["w"], reference(c)[2]
    left = lambda x: 1.0 / (1.0 + np.exp(x))   # one less the sigmoid of x, without a difference
    none = held | {"s": np.zeros_like(held["s"])}   # dgate up to its factor 1 - s
    ref, scale = orc.scan_gradients(w["x"], w["input"], w["rate"], none, w["dout"], w["dstate_out"], reverse)
    steps = 2 * STEPS[dtype] + 8
    near(f64(d["dgate"]), ref["dgate"] * left(w["gate"]), dtype, steps, scale["dgate"] * left(w["gate"]), "dgate")
    if inputs:
        near(f64(d["dinput"]), ref["dx"] * w["x"] * left(w["input"]), dtype, steps, scale["dinput"] * left(w["input"]), "dinput")

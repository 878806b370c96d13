"""Rows of many chunks against fp64: the chain from one group of chunks to the next where many chunks lie side by side, the chain of stretches of
groups where few do, out, states and every gradient, in all types and with all weights of the new value."""
import pytest
import torch

from tests.test_gpu_scan import backward, check_all, forward, make, on_gpu

pytestmark = pytest.mark.gpu


def check(c):
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    check_all(c, out, last, grads)
    again = backward(c, g, None)   # without what the forward pass saved: the same
    assert all(torch.equal(grads[n], again[n]) for n in grads)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight,inputs,state,reverse", [("norm", True, True, False), ("leaky", False, True, True), ("sum", True, False, True)])
@pytest.mark.parametrize("B,N,C,lengths", [(1, 4500, 520, None), (2, 6500, 264, (4096, 6500)), (3, 6500, 200, (4097, 2048, 6143)), (4, 4200, 128, (2049, 0, 2047, 4200))],
                         ids=str)
def test_groups(B, N, C, lengths, weight, inputs, state, reverse, dtype):
    """33 chunks of 128 tokens and more, eight and more side by side: rows of one group of 16 chunks, two, three and four, whole and not."""
    check(make(B, N, C, dtype, N + C, weight, inputs, state, reverse, lengths))


@pytest.mark.parametrize("reverse", [False, True])
def test_more_than_a_group_in_the_widest_rows(reverse):
    check(make(3, 2300, 1280, "bf16", 16, reverse=reverse, lengths=(2300, 1150, 0)))


@pytest.mark.parametrize("dtype,weight,inputs,reverse", [("f16", "norm", True, False), ("bf16", "leaky", True, True), ("f16", "sum", False, True), ("f32", "leaky", False, False),
                                                         ("f32", "sum", True, False)])
def test_stretches(dtype, weight, inputs, reverse):
    """266 chunks, one beside the other: a stretch of 256 of them and a rest."""
    check(make(1, 34000, 16, dtype, 7, weight, inputs, True, reverse))

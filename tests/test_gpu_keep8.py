"""Activations kept in 8 bits on the GPU: bit for bit the oracle's."""
import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import layers_oracle as orc
from tests.layers_parity import TORCH, columns, f64, stored

pytestmark = pytest.mark.gpu


def keep(x, lengths=None):
    codes = torch.full(x.shape, 99, dtype=torch.int8, device="cuda")
    exps = torch.full((*x.shape[:2], (x.shape[2] + 31) // 32), 77, dtype=torch.uint8, device="cuda")
    back = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
    lf.linfusion_keep8(x, codes, exps, lengths=lengths)
    lf.linfusion_unkeep8(codes, exps, back, lengths=lengths)
    return codes, exps, back


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 8), (2, 3, 24), (1, 7, 32), (3, 65, 40), (2, 130, 328), (1, 1000, 64), (5, 9, 1280), (1, 3, 8192)], ids=str)
def test_against_the_oracle(shape, dtype):
    r = np.random.RandomState(sum(shape))
    t, x = stored(r.randn(*shape) * np.exp2(r.randint(-12, 12, shape[:2] + (1,))), dtype)
    codes, exps, back = keep(t.cuda())
    want = orc.keep8(x)
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(exps.cpu().numpy(), want[1])
    assert np.array_equal(f64(back), want[2])
    # off by at most 1 / 127 of the block's largest
    for q in range(0, shape[2], 32):
        most = np.abs(x[..., q:q + 32]).max(-1, keepdims=True)
        assert (np.abs(want[2] - x)[..., q:q + 32] <= most / 127).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_edges(dtype):
    """Zeros, ties, subnormals, the largest values, blocks with an infinity or a NaN, and powers of two around 127."""
    info = torch.finfo(TORCH[dtype])
    x = torch.zeros((1, 14, 64), dtype=TORCH[dtype])
    x[0, 1, :32] = torch.arange(32) * 0.5            # ties, to even
    x[0, 1, 31] = 127.0
    x[0, 2, 0] = info.smallest_normal * info.eps      # the least subnormal
    x[0, 3, :4] = torch.tensor([info.max / 2, -info.max / 2, info.max / 256, 1.0])
    x[0, 4, 5], x[0, 5, 6], x[0, 6, 40] = float("inf"), float("nan"), float("-inf")
    for i, v in enumerate((127.0, 127.5, 128.0, 126.0, 0.99609375, 254.0)):
        x[0, 7 + i, 3] = v
        x[0, 7 + i, 4] = -1.0
    x[0, 13] = info.max
    codes, exps, back = keep(x.cuda())
    want = orc.keep8(x.double().numpy())
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(exps.cpu().numpy(), want[1])
    got, ref = f64(back), np.clip(want[2], -info.max, info.max)
    assert np.array_equal(got, ref, equal_nan=True)
    assert np.isnan(got[0, 4, :32]).all() and np.isnan(got[0, 5, :32]).all() and (got[0, 4, 32:] == 0).all()
    assert (got[0, 13] == info.max).all()


def test_ragged_rows_and_views():
    r = np.random.RandomState(1)
    t, x = stored(r.randn(3, 40, 72), "bf16")
    g = t.cuda()
    lengths = torch.tensor([40, 0, 13], dtype=torch.int32, device="cuda")
    full = keep(g)
    g2 = g.clone()
    g2[1], g2[2, 13:] = float("nan"), float("nan")
    codes, exps, back = keep(g2, lengths)
    for got, whole, none in zip((codes, exps, back), full, (99, 77, 7.0)):
        for b, n in enumerate((40, 0, 13)):
            assert torch.equal(got[b, :n], whole[b, :n]) and bool((got[b, n:] == none).all())
    v, _ = columns([g, g], 8)
    flat = torch.zeros((3, 40, 72 + 8 + 72), dtype=torch.int8, device="cuda")
    e = torch.zeros((3, 40, 7), dtype=torch.uint8, device="cuda")
    lf.linfusion_keep8(v, flat[..., 80:], e[..., 2:5])
    assert torch.equal(flat[..., 80:], full[0]) and torch.equal(e[..., 2:5], full[1])
    assert not flat[..., :80].any() and not e[..., :2].any() and not e[..., 5:].any()
    out, _ = columns([torch.zeros_like(g), torch.zeros_like(g)], 8)
    lf.linfusion_unkeep8(flat[..., 80:], e[..., 2:5], out)
    assert torch.equal(out, full[2])

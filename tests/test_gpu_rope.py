"""Rotary positions with several axes on the GPU against fp64."""
import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import block_oracle as orc
from tests.block_parity import TORCH, check, f64, stored

pytestmark = pytest.mark.gpu

# sine and cosine: the library's to 4 steps of fp32 for fp32; the hardware's, whose argument is rounded to 2^-25 turns (2^-22.3 in the
# angle) and whose result to about 2^-20, for the 16-bit types.  Two products and a sum: 3 steps more.
STEPS = {"f32": 2 * (4 + 2) + 3, "f16": 2 * (16 + 4) + 3, "bf16": 2 * (16 + 4) + 3}


def make(B, H, Hk, N, d, dtype, seed):
    r = np.random.RandomState(seed)
    q, k = (stored(r.randn(B, h, N, d), dtype) for h in (H, Hk))
    return q[0], q[1], k[0], k[1], r


def as_tokens(t):
    return t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("shape,channels", [
    ((1, 1, 1, 1, 8), (8,)), ((2, 3, 1, 37, 40), (20, 20)), ((1, 8, 8, 200, 40), (16, 16)), ((2, 4, 4, 65, 64), (16, 24, 24)),
    ((1, 5, 5, 33, 80), (32, 48)), ((1, 2, 1, 130, 128), (44, 42, 42)), ((1, 2, 2, 77, 160), (80, 80)), ((1, 1, 1, 50, 256), (64, 64, 64, 64)),
    ((3, 2, 2, 19, 24), (2, 4, 6)), ((1, 4, 2, 500, 64), (64,)),
], ids=str)
def test_against_the_oracle(shape, channels, neighbours, dtype):
    B, H, Hk, N, d = shape
    q, wq, k, wk, r = make(*shape, dtype, sum(shape))
    pos = r.randint(-5, 3000, (B, len(channels), N)).astype(np.int32)
    bases = [1e4, 100.0, 5e5, 1.0][:len(channels)]
    scales = [1.0, 0.37, 2.0, 1.0][:len(channels)]
    flags = lf.FLAG_ROPE_NEIGHBOURS if neighbours else 0
    gp = torch.from_numpy(pos).cuda()
    for inverse in (False, True):
        gq, gk = as_tokens(q), k.cuda()
        oq, ok = torch.full_like(gq, float("nan")), torch.full_like(gk, float("nan"))
        lf.linfusion_rope(gq, gk, oq, ok, gp, channels, bases, scales, flags=flags | (lf.FLAG_ROPE_INVERSE if inverse else 0))
        for got, x, name in ((oq, wq, "q"), (ok, wk, "k")):
            check(got, orc.rope(x, pos, channels, bases, scales, neighbours, inverse), dtype, STEPS[dtype], f"{name} inverse={inverse}")
        rest = sum(channels)
        assert torch.equal(oq[..., rest:], gq[..., rest:]) and torch.equal(ok[..., rest:], gk[..., rest:])
        lf.linfusion_rope(gq, gk, gq, gk, gp, channels, bases, scales, flags=flags | (lf.FLAG_ROPE_INVERSE if inverse else 0))
        assert torch.equal(gq, oq) and torch.equal(gk, ok)   # in place


def test_far_positions_in_fp32():
    q, wq, k, wk, r = make(1, 2, 2, 64, 64, "f32", 3)
    pos = (2 ** 30 + r.randint(0, 2 ** 30, (2, 64))).astype(np.int32)
    gq, gk = q.cuda(), k.cuda()
    lf.linfusion_rope(gq, gk, gq, gk, torch.from_numpy(pos).cuda(), (32, 32), (1e4, 1e4))
    # the fp64 angle of 2^31 is exact to 2^-22 steps of a turn on both sides: 2^31 2^-53, twelve times fp32's step
    check(gq, orc.rope(wq, pos, (32, 32), (1e4, 1e4)), "f32", STEPS["f32"] + 2 * 16, "q")


def test_queries_alone_and_lengths():
    lengths = [0, 1, 40, 99]
    q, wq, _, _, r = make(4, 3, 1, 40, 40, "bf16", 5)
    q[0] = float("nan")
    q[1, :, 1:] = float("inf")
    pos = np.arange(40, dtype=np.int32)[None]
    gq = as_tokens(q)
    out = torch.full_like(gq, 3.0)
    lf.linfusion_rope(gq, None, out, None, torch.from_numpy(pos).cuda(), (40,), (1e4,),
                      lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    ref = orc.rope(wq, pos, (40,), (1e4,))
    for b, n in enumerate(lengths):
        n = min(n, 40)
        assert bool((out[b, :, n:] == 3.0).all())
        check(out[b, :, :n], ref[b, :, :n], "bf16", STEPS["bf16"], f"row {b}", scale=np.abs(wq).max())


def test_columns_of_one_projection_in_place():
    """Queries and keys as column blocks of one [B, N, 3, H, d] projection, turned where they are; the values stay."""
    B, N, H, d = 2, 50, 4, 32
    r = np.random.RandomState(9)
    x, wx = stored(r.randn(B, N, 3, H, d), "f16")
    gx = x.cuda()
    q, k = (gx[:, :, i].permute(0, 2, 1, 3) for i in (0, 1))
    pos = np.stack([np.arange(N) // 10, np.arange(N) % 10]).astype(np.int32)
    lf.linfusion_rope(q, k, q, k, torch.from_numpy(pos).cuda(), (16, 16), (1e4, 1e4))
    for i, t in ((0, q), (1, k)):
        check(t, orc.rope(wx[:, :, i].transpose(0, 2, 1, 3), pos, (16, 16), (1e4, 1e4)), "f16", STEPS["f16"], str(i))
    assert torch.equal(gx[:, :, 2].cpu(), x[:, :, 2])
    with pytest.raises(lf.LinFusionError):   # keys that overlap the queries
        lf.linfusion_rope(q, q, q, q, torch.from_numpy(pos).cuda(), (16, 16), (1e4, 1e4))


def test_turning_there_and_back_and_the_gradient():
    q, wq, _, _, r = make(1, 2, 1, 100, 48, "f32", 7)
    pos = torch.from_numpy(r.randint(0, 500, (2, 100)).astype(np.int32)).cuda()
    gq = q.cuda()
    out = torch.empty_like(gq)
    lf.linfusion_rope(gq, None, out, None, pos, (24, 24), (1e4, 1e4))
    up, wup = stored(r.randn(1, 2, 100, 48), "f32")
    dq = torch.empty_like(gq)
    lf.linfusion_rope(up.cuda(), None, dq, None, pos, (24, 24), (1e4, 1e4), flags=lf.FLAG_ROPE_INVERSE)
    # <rope(q), up> = <q, dq>, the defining property of a linear map's gradient
    left, right = (f64(out) * wup).sum(), (wq * f64(dq)).sum()
    assert abs(left - right) <= 2 * STEPS["f32"] * 2.0 ** -24 * np.abs(wq * f64(dq)).sum()
    lf.linfusion_rope(out, None, out, None, pos, (24, 24), (1e4, 1e4), flags=lf.FLAG_ROPE_INVERSE)
    check(out, wq, "f32", 2 * STEPS["f32"], "there and back")


def test_graph_and_other_stream():
    q, wq, k, wk, r = make(1, 4, 4, 300, 64, "bf16", 1)
    gq, gk = as_tokens(q), as_tokens(k)
    oq, ok = torch.empty_like(gq), torch.empty_like(gk)
    pos = torch.stack([torch.arange(300) // 20, torch.arange(300) % 20]).int().cuda()
    call = lambda: lf.linfusion_rope(gq, gk, oq, ok, pos, (32, 32), (1e4, 1e4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    want = oq.clone(), ok.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        oq.fill_(0)
        ok.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])


def test_offsets_past_32_bits():
    q, wq, _, _, r = make(2, 1, 1, 20, 16, "bf16", 2)
    far = (1 << 31) + 64
    big = torch.empty(far + 320, dtype=torch.bfloat16, device="cuda").as_strided((2, 1, 20, 16), (far, 320, 16, 1))
    big.copy_(q)
    pos = np.arange(20, dtype=np.int32)[None]
    lf.linfusion_rope(big, None, big, None, torch.from_numpy(pos).cuda(), (16,), (1e4,))
    check(big, orc.rope(wq, pos, (16,), (1e4,)), "bf16", STEPS["bf16"], "q")


def test_refusals_on_the_device():
    x = torch.zeros(1, 2, 10, 32, device="cuda")
    pos = torch.zeros(1, 10, dtype=torch.int32, device="cuda")
    for bad in (dict(positions=pos.long()), dict(positions=pos[:, :5]), dict(channels=(16, 16)), dict(q=x.transpose(2, 3)),
                dict(q_out=x.half()), dict(q=x.cpu())):
        a = dict(q=x, k=None, q_out=x, k_out=None, positions=pos, channels=(32,), bases=(1e4,)) | bad
        with pytest.raises(ValueError):
            lf.linfusion_rope(**a)


@pytest.mark.parametrize("B,N,per_head", [(5, 1, False), (2, 1, True), (3, 30, True)])
def test_interleaved_views_in_place(B, N, per_head):
    """Queries and keys of one projection turned where they are: a token for each of several users, and the parts head by head."""
    H, d = 4, 32
    r = np.random.RandomState(10)
    x, wx = stored(r.randn(*((B, N, H, 3, d) if per_head else (B, N, 3, H, d))), "bf16")
    gx = x.cuda()
    part = lambda t, i: t[:, :, :, i] if per_head else t[:, :, i]
    q, k = (part(gx, i).permute(0, 2, 1, 3) for i in (0, 1))
    pos = r.randint(0, 1000, (B, 1, N)).astype(np.int32)
    lf.linfusion_rope(q, k, q, k, torch.from_numpy(pos).cuda(), (32,), (1e4,))
    for i, t in ((0, q), (1, k)):
        check(t, orc.rope(part(wx, i).transpose(0, 2, 1, 3), pos, (32,), (1e4,)), "bf16", STEPS["bf16"], str(i))
    assert torch.equal(part(gx, 2).cpu(), part(x, 2))


def test_rows_of_many_more_tokens_than_workgroups():
    """2^24 tokens and more of 16 KB are within the documented range; a row's length says that three of them are there."""
    import ctypes
    H, d, far = 32, 256, (1 << 24) + 5
    q, wq, _, _, _ = make(1, H, 1, 3, d, "bf16", 11)
    at = 256 + (4 * far + 255) // 256 * 256   # (what is read lies before the view that ends nowhere: a length, positions of all tokens)
    room = torch.empty(at + 3 * H * d * 2, dtype=torch.uint8, device="cuda")
    lengths, pos = room[:256].view(torch.int32), room[256:at].view(torch.int32)
    pos[:3] = torch.arange(3)
    lengths[0] = 3
    gq = room[at:].view(torch.bfloat16).view(1, 3, H, d).permute(0, 2, 1, 3)
    gq.copy_(q)
    strides = (ctypes.c_longlong * 3)(0, d, H * d)
    rc = lf.library().linfusion_rope(gq.data_ptr(), None, gq.data_ptr(), None, pos.data_ptr(), 1, (ctypes.c_int * 1)(d), (ctypes.c_double * 1)(1e4), None, 1, H,
                                     0, far, d, lf.DTYPE_BF16, 0, lengths.data_ptr(), strides, None, strides, None, None,
                                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0
    check(gq, orc.rope(wq, np.arange(3)[None], (d,), (1e4,)), "bf16", STEPS["bf16"], "q")


def test_outputs_beside_their_inputs():
    B, N, H, d = 2, 70, 3, 40
    r = np.random.RandomState(12)
    x, wx = stored(r.randn(B, N, 5, H, d), "f16")
    gx = x.cuda()
    q, k, qo, ko = (gx[:, :, i].permute(0, 2, 1, 3) for i in range(4))
    pos = r.randint(0, 1000, (2, N)).astype(np.int32)
    lf.linfusion_rope(q, k, qo, ko, torch.from_numpy(pos).cuda(), (16, 20), (1e4, 1e4))
    for i, t in ((0, qo), (1, ko)):
        check(t, orc.rope(wx[:, :, i].transpose(0, 2, 1, 3), pos, (16, 20), (1e4, 1e4)), "f16", STEPS["f16"], str(i))
    for i in (0, 1, 4):
        assert torch.equal(gx[:, :, i].cpu(), x[:, :, i])

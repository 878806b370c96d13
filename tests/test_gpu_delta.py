"""The gated delta rule on the GPU against the fp64 recurrence: forward, gradients, single tokens."""
import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import block_oracle as orc
from tests.block_parity import TORCH, check, f64, stored
from tests.delta_bounds import excess, references

pytestmark = pytest.mark.gpu

CODE = {"f32": lf.DTYPE_F32, "f16": lf.DTYPE_F16, "bf16": lf.DTYPE_BF16}


def make(B, H, Hk, N, dk, dv, dtype, seed, state=True, lengths=None):
    r = np.random.RandomState(seed)
    unit = lambda x: x / np.sqrt((x * x).sum(-1, keepdims=True))
    c = {"dtype": dtype, "scale": dk ** -0.5, "dims": (B, H, Hk, N, dk, dv)}
    wide = {"q": unit(r.randn(B, Hk, N, dk) + 0.3), "k": unit(r.randn(B, Hk, N, dk) + 0.3), "v": r.randn(B, H, N, dv),
            "dout": r.randn(B, H, N, dv)}
    c["cpu"] = {}
    for n, x in wide.items():
        c["cpu"][n], c[n] = stored(x, dtype)
    scalars = {"g": -np.exp(r.uniform(-7, 0.5, (B, H, N))), "beta": r.uniform(0, 1, (B, H, N)),
               "state": 0.3 * r.randn(B, H, dk, dv), "dstate": 0.1 * r.randn(B, H, dk, dv)}
    for n, x in scalars.items():
        c["cpu"][n], c[n] = stored(x, "f32")
    if not state:
        c["state"] = c["dstate"] = c["cpu"]["state"] = c["cpu"]["dstate"] = None
    c["lengths"] = lengths
    return c


def on_gpu(c, tokens=True):
    """The case's tensors on the GPU; `tokens`: rows as views of [B, N, heads, d] activations."""
    g = {}
    for n, t in c["cpu"].items():
        if t is None:
            g[n] = None
        elif n in ("q", "k", "v", "dout") and tokens:
            g[n] = t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
        elif n in ("g", "beta") and tokens:
            g[n] = t.permute(0, 2, 1).contiguous().cuda().permute(0, 2, 1)
        else:
            g[n] = t.cuda()
    g["lengths"] = None if c["lengths"] is None else torch.tensor(c["lengths"], dtype=torch.int32, device="cuda")
    return g


def forward(c, g, saved=False, fill=0.0):
    B, H, Hk, N, dk, dv = c["dims"]
    out = torch.full_like(g["v"], fill)
    last = torch.full((B, H, dk, dv), float("nan"), device="cuda")
    size = (lf.linfusion_delta_saved_bytes if saved else lf.linfusion_delta_workspace_bytes)(*c["dims"][:3], N, dk, dv, CODE[c["dtype"]])
    mem = torch.full((size,), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever nothing was written)
    lf.linfusion_delta_fwd(g["q"], g["k"], g["v"], g["g"], g["beta"], out, scale=c["scale"], state_in=g["state"], state_out=last,
                           lengths=g["lengths"], saved=mem if saved else None, workspace=None if saved else mem)
    return out, last, mem


def backward(c, g, saved=None, fill=0.0, into=None):
    B, H, Hk, N, dk, dv = c["dims"]
    names = ("q", "k", "v", "g", "beta")
    d = into or {n: torch.full_like(g[n], fill) for n in names}
    d["state"] = torch.full((B, H, dk, dv), float("nan"), device="cuda")
    size = lf.linfusion_delta_bwd_workspace_bytes(B, H, Hk, N, dk, dv, CODE[c["dtype"]])
    if saved is not None:
        size -= saved.numel()
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    lf.linfusion_delta_bwd(g["q"], g["k"], g["v"], g["g"], g["beta"], g["dout"], *(d[n] for n in names), scale=c["scale"],
                           state_in=g["state"], dstate_out=g["dstate"], dstate_in=d["state"], lengths=g["lengths"], saved=saved,
                           workspace=ws)
    return d


def chain(c):
    """Lengths of the longest chains of sums: scores over d_k, the solve and the sums within a chunk over 64, the products with a
    state over d_k or d_v; what a state carries on from earlier chunks shrinks there."""
    dk, dv = c["dims"][4:]
    return 3 * (64 + dk + dv)


def oracle(c):
    return orc.delta(c["q"], c["k"], c["v"], c["g"], c["beta"], c["scale"], c["state"], c["lengths"])


def check_forward(c, out, last):
    ref, end, _ = oracle(c)
    check(out, ref, c["dtype"], chain(c), "out")
    check(last, end, "f32", chain(c), "state")


def check_backward(c, d):
    B, H, Hk, N, dk, dv = c["dims"]
    _, last, held = oracle(c)
    ref = orc.delta_gradients(c["q"], c["k"], c["v"], c["g"], c["beta"], c["scale"], held, c["dout"], c["dstate"], c["lengths"])
    n, group = chain(c), H // Hk
    # sums of terms: dq, dk, dbeta and dv of the largest token; dg is a difference of sums over a chunk's tokens, of the
    # q.dq and v.dv of single value heads, and of the state's product with its gradient
    for name, r in zip(("q", "k", "v"), ref):
        check(d[name], r, c["dtype"], n * group, "d" + name)
    check(d["beta"], ref[4], "f32", n, "dbeta", scale=max(np.abs(ref[4]).max(), np.abs(ref[2]).max() * np.sqrt(dv)))
    each = orc.delta_gradients(np.repeat(c["q"], group, 1), np.repeat(c["k"], group, 1), c["v"], c["g"], c["beta"], c["scale"], held,
                               c["dout"], c["dstate"], c["lengths"])
    terms = np.abs(np.repeat(c["q"], group, 1) * each[0]).sum(-1) + np.abs(c["v"] * each[2]).sum(-1)
    check(d["g"], ref[3], "f32", n, "dg", scale=max(np.abs(ref[3]).max(), terms.max() * 8))
    check(d["state"], ref[5], "f32", n, "dstate")


SHAPES = [
    (1, 1, 1, 1, 8, 8), (2, 2, 1, 2, 16, 24), (1, 2, 2, 63, 40, 40), (1, 2, 2, 64, 64, 64), (2, 2, 1, 65, 24, 72),
    (1, 3, 3, 130, 80, 80), (1, 2, 1, 197, 96, 64), (2, 4, 2, 129, 128, 128), (1, 2, 2, 200, 160, 160), (1, 1, 1, 70, 8, 256),
    (1, 4, 1, 257, 32, 48),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_gradients(shape, dtype):
    c = make(*shape, dtype, seed=sum(shape), state=shape[3] % 2 == 1)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_saved_and_contiguous_the_same_bits(dtype):
    c = make(2, 4, 2, 150, 40, 56, dtype, seed=11)
    g, flat = on_gpu(c), on_gpu(c, tokens=False)
    out, last, saved = forward(c, g, saved=True)
    again = forward(c, flat)
    assert torch.equal(out, again[0]) and torch.equal(last, again[1])
    d, e = backward(c, g, saved), backward(c, flat)
    for n in d:
        assert torch.equal(d[n], e[n]), n
    d = backward(c, g, saved)   # and run to run
    for n in d:
        assert torch.equal(d[n], e[n]), n


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_lengths(dtype):
    """Rows of every length; what stands behind them is not read (NaN, infinity) and left as it was."""
    N, lengths = 140, [0, 1, 64, 65, 139, 140, 9999, -3]
    c = make(8, 2, 1, N, 24, 40, dtype, seed=5, lengths=lengths)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), N)
        for name, bad in (("q", float("nan")), ("k", float("inf")), ("v", float("nan")), ("dout", float("nan"))):
            c["cpu"][name][b, :, n:] = bad
        c["cpu"]["g"][b, :, n:] = float("nan")
        c["cpu"]["beta"][b, :, n:] = float("inf")
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True, fill=7.0)
    d = backward(c, g, saved, fill=7.0)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), N)
        for t in (out, d["q"], d["k"], d["v"], d["g"], d["beta"]):
            assert bool((t[b, :, n:] == 7.0).all())
            t[b, :, n:] = 0.0
    check_forward(c, out, last)
    check_backward(c, d)


def test_decays_and_corrections_at_their_ends():
    """g = 0, -infinity and far below what fp32 holds of exp; beta = 0, 1, and 2 with unit keys."""
    c = make(1, 2, 2, 150, 32, 32, "f32", seed=21)
    for i, v in ((3, -np.inf), (4, 0.0), (64, -np.inf), (65, -300.0), (100, -1e30), (101, -90.0), (149, -np.inf)):
        c["g"][:, :, i] = v
    c["beta"][:, :, 10:20] = 0.0
    c["beta"][:, :, 64] = 0.0
    c["beta"][:, :, 20] = 1.0
    c["beta"][:, :, 30] = 2.0
    c["cpu"]["g"], c["cpu"]["beta"] = (torch.from_numpy(c[n]).float() for n in ("g", "beta"))
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved))


def test_nothing_corrected_is_nothing_kept():
    c = make(1, 2, 2, 100, 16, 16, "f32", seed=1, state=False)
    c["cpu"]["beta"].zero_()
    g = on_gpu(c)
    out, last, _ = forward(c, g)
    assert bool((out == 0).all()) and bool((last == 0).all())


def test_small_decays_behind_a_large_one():
    """Differences of an fp32 running sum behind g = -1e4 would be off by 5e-4."""
    c = make(1, 1, 1, 64, 16, 16, "f32", seed=2)
    c["g"][:] = -0.01
    c["g"][:, :, 2] = -9000.0
    c["cpu"]["g"] = torch.from_numpy(c["g"]).float()
    c["g"] = c["cpu"]["g"].double().numpy()
    out, last, _ = forward(c, on_gpu(c))
    check_forward(c, out, last)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_sequence_in_pieces(dtype):
    c = make(1, 2, 1, 210, 40, 64, dtype, seed=8)
    g = on_gpu(c)
    state, outs = g["state"].clone(), []
    for lo, hi in ((0, 70), (70, 71), (71, 199), (199, 210)):
        out = torch.empty_like(g["v"][:, :, lo:hi])
        ws = torch.empty(lf.linfusion_delta_workspace_bytes(1, 2, 1, hi - lo, 40, 64, CODE[dtype]), dtype=torch.uint8, device="cuda")
        cut = {n: g[n][:, :, lo:hi] for n in ("q", "k", "v", "g", "beta")}
        lf.linfusion_delta_fwd(*cut.values(), out, scale=c["scale"], state_in=state, state_out=state, workspace=ws)
        outs.append(out)
    check_forward(c, torch.cat(outs, 2), state)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 8, 8), (3, 4, 2, 40, 24), (2, 2, 2, 64, 64), (1, 4, 1, 128, 136), (2, 2, 1, 160, 256)], ids=str)
def test_single_tokens(shape, dtype):
    """Eight tokens one by one, the state in place; the same values as the whole sequence."""
    B, H, Hk, dk, dv = shape
    c = make(B, H, Hk, 8, dk, dv, dtype, seed=sum(shape))
    g = on_gpu(c)
    state, out = g["state"].clone(), torch.full_like(g["v"], float("nan"))
    for t in range(8):
        lf.linfusion_delta_step(*(g[n][:, :, t] for n in ("q", "k", "v", "g", "beta")), state, state, out[:, :, t], scale=c["scale"])
    check_forward(c, out, state)


def test_single_token_without_a_state():
    c = make(2, 2, 2, 1, 32, 32, "f32", seed=3, state=False)
    g = on_gpu(c)
    out, last = torch.empty_like(g["v"]), torch.empty((2, 2, 32, 32), device="cuda")
    lf.linfusion_delta_step(*(g[n][:, :, 0] for n in ("q", "k", "v", "g", "beta")), None, last, out[:, :, 0], scale=c["scale"])
    check_forward(c, out, last)


def test_shared_inputs_by_stride_zero():
    """One key sequence for all batch rows and heads."""
    c = make(2, 2, 2, 90, 24, 24, "f32", seed=13)
    c["cpu"]["k"] = c["cpu"]["k"][:1, :1].expand(2, 2, 90, 24)
    c["k"] = c["cpu"]["k"].double().numpy()
    g = on_gpu(c, tokens=False)
    g["k"] = g["k"][:1, :1].contiguous().expand(2, 2, 90, 24)
    assert g["k"].stride()[:2] == (0, 0)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved, into={n: torch.empty((2, 2, 90, 24), device="cuda") for n in "qkv"}
                               | {n: torch.empty((2, 2, 90), device="cuda") for n in ("g", "beta")}))


def test_gradients_against_differences():
    """Along a random direction of every input the gradient's product with it is the loss's slope in the fp64 oracle."""
    c = make(1, 2, 1, 75, 16, 24, "f32", seed=31)
    d = backward(c, on_gpu(c))
    loss = lambda c: (lambda o: (o[0] * c["dout"]).sum() + (o[1] * c["dstate"]).sum())(oracle(c))
    r, eps = np.random.RandomState(4), 1e-5
    for name in ("q", "k", "v", "g", "beta", "state"):
        way = r.randn(*c[name].shape)
        slope = (loss(dict(c, **{name: c[name] + eps * way})) - loss(dict(c, **{name: c[name] - eps * way}))) / (2 * eps)
        terms = f64(d[name]) * way
        # the differences are exact to about eps^2 and 1e-16 / eps of the loss; the gradient to its own bound per element
        assert abs(terms.sum() - slope) <= 1e-6 * np.abs(terms).sum() + chain(c) * 2.0 ** -24 * np.abs(terms).sum(), name


def test_captured_and_replayed_beside_other_work():
    c = make(2, 4, 2, 200, 64, 64, "bf16", seed=17)
    g = on_gpu(c)
    want, last, saved = forward(c, g, saved=True)
    grads = backward(c, g, saved)
    out, end = torch.empty_like(want), torch.empty_like(last)
    d = {n: torch.empty_like(g[n]) for n in ("q", "k", "v", "g", "beta")}
    dstate = torch.empty_like(end)
    ws = torch.empty(lf.linfusion_delta_bwd_workspace_bytes(2, 4, 2, 200, 64, 64, CODE["bf16"]), dtype=torch.uint8, device="cuda")

    def both():
        lf.linfusion_delta_fwd(g["q"], g["k"], g["v"], g["g"], g["beta"], out, scale=c["scale"], state_in=g["state"], state_out=end,
                               saved=saved)
        lf.linfusion_delta_bwd(g["q"], g["k"], g["v"], g["g"], g["beta"], g["dout"], *d.values(), scale=c["scale"],
                               state_in=g["state"], dstate_out=g["dstate"], dstate_in=dstate, saved=saved, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for t in (out, end, dstate, *d.values(), saved, ws):
            t.view(torch.uint8).reshape(-1).fill_(255) if t.is_contiguous() else t.fill_(float("nan"))
        torch.randn(1 << 20, device="cuda").sum()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(end, last) and torch.equal(dstate, grads["state"])
        for n in d:
            assert torch.equal(d[n], grads[n]), n


def test_offsets_past_32_bits():
    """Two batch rows more than 2^32 bytes and 2^31 elements apart."""
    c = make(2, 1, 1, 70, 16, 16, "bf16", seed=41)
    g = on_gpu(c, tokens=False)
    far = (1 << 31) + 64
    for n in ("q", "k", "v"):
        big = torch.empty(far + 70 * 16, dtype=torch.bfloat16, device="cuda").as_strided((2, 1, 70, 16), (far, 70 * 16, 16, 1))
        big.copy_(g[n])
        g[n] = big
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)


def test_refusals_on_the_device():
    c = make(1, 2, 1, 70, 16, 16, "f32", seed=1)
    g = on_gpu(c)
    out = torch.empty_like(g["v"])
    ws = torch.empty(lf.linfusion_delta_workspace_bytes(1, 2, 1, 70, 16, 16, lf.DTYPE_F32), dtype=torch.uint8, device="cuda")
    call = lambda **kw: lf.linfusion_delta_fwd(*({n: g[n] for n in ("q", "k", "v", "g", "beta")} | kw).values(), out, workspace=ws)
    with pytest.raises(ValueError):
        call(k=g["k"].to(torch.bfloat16))
    with pytest.raises(ValueError):
        call(g=g["g"].contiguous())            # other strides than beta's
    with pytest.raises(ValueError):
        call(q=g["q"].transpose(2, 3))
    with pytest.raises(ValueError):
        call(v=g["v"].cpu())
    with pytest.raises(lf.LinFusionError) as e:
        lf.linfusion_delta_fwd(g["q"], g["k"], g["v"], g["g"], g["beta"], out, workspace=ws[:-256])
    assert e.value.status == -4
    with pytest.raises(lf.LinFusionError) as e:
        lf.linfusion_delta_fwd(g["q"], g["k"], g["v"], g["g"], g["beta"], g["v"], workspace=ws)
    assert e.value.status == -7


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 40, 24), ("f32", 16, 16), ("f16", 72, 40)])
def test_long_sequences_of_few_heads_in_runs(dtype, dk, dv):
    """Chunks parted into runs, whole and not, rows that end inside each of them; gradients behind such a forward call."""
    N, lengths = 64 * 70 + 5, [64 * 70 + 5, 64 * 33, 1100, 0]
    c = make(4, 1, 1, N, dk, dv, dtype, seed=51, lengths=lengths)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    d = backward(c, g, saved)
    for b, n in enumerate(lengths):
        for t in (out, *(d[m] for m in ("q", "k", "v", "g", "beta"))):
            t[b, :, n:] = 0.0
    check_forward(c, out, last)
    check_backward(c, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_heads(dtype):
    """Enough heads for 32 value channels a workgroup, an odd number of 16s among them."""
    c = make(16, 8, 8, 70, 16, 40, dtype, seed=61)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved))


def test_runs_of_many_heads():
    """Runs whose first pass takes 32 channels a workgroup too."""
    B, H, N, d = 1, 8, 64 * 220 - 7, 32
    c = make(B, H, H, N, d, d, "bf16", seed=62)
    g = on_gpu(c)
    out, last, _ = forward(c, g)
    ref = np.zeros((B, H, N, d))
    s = np.array(c["state"])
    for t in range(N):   # (all heads at once; the states of all tokens would be a gigabyte)
        key, qry = c["k"][:, :, t], c["q"][:, :, t]
        s *= np.exp(c["g"][:, :, t])[..., None, None]
        u = c["beta"][:, :, t, None] * (c["v"][:, :, t] - np.matmul(key[:, :, None], s)[:, :, 0])
        s += key[..., None] * u[:, :, None]
        ref[:, :, t] = c["scale"] * np.matmul(qry[:, :, None], s)[:, :, 0]
    check(out, ref, "bf16", chain(c), "out")
    check(last, s, "f32", chain(c), "state")


def test_two_graphs_that_share_a_workspace_and_a_stream_of_their_own():
    cases = [make(2, 4, 2, 130, 40, 56, "bf16", seed=71), make(2, 4, 2, 130, 40, 56, "bf16", seed=72)]
    gs = [on_gpu(c) for c in cases]
    want = [forward(c, g) for c, g in zip(cases, gs)]
    ws = torch.empty(lf.linfusion_delta_workspace_bytes(2, 4, 2, 130, 40, 56, CODE["bf16"]), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(w[0]) for w in want]
    call = lambda i, **kw: lf.linfusion_delta_fwd(*(gs[i][n] for n in ("q", "k", "v", "g", "beta")), outs[i], scale=cases[i]["scale"],
                                                  state_in=gs[i]["state"], workspace=ws, **kw)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(0, stream=side)          # named, not current
    side.synchronize()
    assert torch.equal(outs[0], want[0][0])
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i)
    for _ in range(3):
        for i in (0, 1, 1, 0):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i][0])


def test_runs_with_the_state_in_place():
    """Rows that end in the first run, just behind it and in the last one: whichever run writes the state, the first has read it."""
    N, lengths = 64 * 70, [64 * 70, 64 * 18 + 1, 64 * 17, 64 * 16, 64, 1, 0, 64 * 40]
    c = make(8, 1, 1, N, 32, 48, "bf16", seed=81, lengths=lengths)
    g = on_gpu(c)
    out, last, mem = forward(c, g)
    again, state = torch.zeros_like(out), g["state"].clone()
    lf.linfusion_delta_fwd(*(g[n] for n in ("q", "k", "v", "g", "beta")), again, scale=c["scale"], state_in=state, state_out=state,
                           lengths=g["lengths"], workspace=mem)
    assert torch.equal(again, out) and torch.equal(state, last)


@pytest.mark.parametrize("dk,dv", [(160, 24), (128, 64)])
def test_runs_of_wide_keys(dk, dv):
    """Three and two blocks of state rows a wave where runs are joined."""
    c = make(1, 2, 1, 64 * 60 + 3, dk, dv, "bf16", seed=91)
    g = on_gpu(c)
    out, last, _ = forward(c, g)
    check_forward(c, out, last)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_corrected_key_answers_its_value(dtype):
    """Unit keys that are columns of the identity, beta = 1, no decay: a token's correction is its value less what the state holds
    for the key, and a query of that key gets the value back, the small rest of two sums of 2^14 and more.

    A row's correction: three products (the terms of the state) and a difference, each rounded to 2^-24 of at most 2^15.  An output:
    three products with the state, three with the correction.  A later chunk's state: three products and a sum more, and its own
    correction again.  Together no more than 18 roundings."""
    N, d, dv = 70, 64, 48
    c = make(1, 2, 2, N, d, dv, dtype, seed=7)
    r = np.random.RandomState(8)
    eye = np.eye(d)
    c["cpu"]["k"], c["k"] = stored(np.broadcast_to(eye[np.arange(N) % d], (1, 2, N, d)), dtype)
    asked = np.array([r.randint(0, min(t, d - 1) + 1) for t in range(N)])
    c["cpu"]["q"], c["q"] = stored(np.broadcast_to(eye[asked], (1, 2, N, d)), dtype)
    c["cpu"]["state"], c["state"] = stored(r.uniform(2.0 ** 14, 2.0 ** 15, (1, 2, d, dv)) * r.choice((-1, 1), (1, 2, d, dv)), "f32")
    for n, x in (("g", np.zeros((1, 2, N))), ("beta", np.ones((1, 2, N)))):
        c["cpu"][n], c[n] = stored(x, "f32")
    c["scale"] = 1.0
    out, _, _ = forward(c, on_gpu(c))
    ref = oracle(c)[0]
    assert np.abs(ref).max() < 8
    check(out, ref, dtype, 18, "out", scale=2.0 ** 15)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,N", [(4, 2, 130), (2, 2, 1)], ids=str)
def test_columns_of_one_buffer(H, Hk, N, dtype):
    """Outputs beside q, k and v in one [B, N, ...] buffer, and their gradients beside each other in another, as those of the scalars: the
    bits of tensors of their own, and nothing else written."""
    B, dk, dv = 2, 40, 56
    c = make(B, H, Hk, N, dk, dv, dtype, seed=19)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    d = backward(c, g, saved)
    widths = (Hk * dk, Hk * dk, H * dv, H * dv, 8)
    room, droom = (torch.full((B, N, sum(widths)), 3.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    scalars = torch.full((B, N, 2 * H + 1), 3.0, device="cuda")
    cut = lambda t: [p.unflatten(-1, (-1, w)).permute(0, 2, 1, 3) for p, w in zip(t.split(widths, -1), (dk, dk, dv, dv, 8))]
    q, k, v, o, _ = cut(room)
    for to, n in ((q, "q"), (k, "k"), (v, "v")):
        to.copy_(g[n])
    packed = dict(g, q=q, k=k, v=v)
    end = torch.empty_like(last)
    lf.linfusion_delta_fwd(q, k, v, g["g"], g["beta"], o, scale=c["scale"], state_in=g["state"], state_out=end, saved=torch.empty_like(saved))
    assert torch.equal(o, out) and torch.equal(end, last)
    dq, dk_, dv_, _, spare = cut(droom)
    into = {"q": dq, "k": dk_, "v": dv_, "g": scalars[..., :H].permute(0, 2, 1), "beta": scalars[..., H:2 * H].permute(0, 2, 1)}
    backward(c, packed, saved, into=into)
    for n in ("q", "k", "v", "g", "beta"):
        assert torch.equal(into[n], d[n]), n
        assert n not in packed or n in ("g", "beta") or torch.equal(packed[n], g[n])
    assert bool((cut(room)[4] == 3.0).all()) and bool((spare == 3.0).all()) and bool((scalars[..., 2 * H] == 3.0).all())
    if N == 1:
        o.fill_(float("nan"))
        lf.linfusion_delta_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], g["g"][:, :, 0], g["beta"][:, :, 0], g["state"], end, o[:, :, 0], scale=c["scale"])
        check_forward(c, o, end)


@pytest.mark.parametrize("shape", [(1, 1, 1, 130, 64, 64), (1, 1, 1, 200, 32, 128), (1, 4, 2, 130, 64, 64), (2, 2, 2, 150, 128, 128), (1, 4, 1, 100, 40, 56),
                                   (1, 2, 1, 90, 160, 40), (1, 2, 1, 90, 96, 96)], ids=str)
def test_whole_gradients_in_fp32(shape):
    """In the 2-norm, where an operand kept to 16 bits shows (test_delta_bounds.py)."""
    c = make(*shape, "f32", seed=sum(shape) + 1)
    d = backward(c, on_gpu(c))
    worst = excess(c, {n: f64(d[n]) for n in ("q", "k", "v", "g", "beta")}, *references(c))
    assert max(worst.values()) <= 1, worst


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dk", [40, 64, 96, 128, 160])
def test_many_heads_of_every_width(dk, dtype):
    """Enough heads for scans of 32 value channels: 3 workgroups for the 5 blocks of 72 channels, 64 heads; more than one chunk."""
    c = make(8, 8, 8, 70, dk, 72, dtype, seed=dk)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dk,dv,group", [(40, 56, 2), (64, 128, 2), (64, 64, 4), (160, 24, 2), (136, 40, 3)])
def test_gradients_summed_over_shared_keys(dk, dv, group, dtype):
    c = make(2, 2 * group, 2, 130, dk, dv, dtype, seed=dk + dv + group)
    g = on_gpu(c)
    out, last, saved = forward(c, g, saved=True)
    check_forward(c, out, last)
    check_backward(c, backward(c, g, saved))


@pytest.mark.parametrize("dtype,dk,dv", [("f32", 64, 64), ("f32", 128, 64), ("f32", 160, 24), ("f16", 128, 40), ("f32", 96, 48)])
def test_runs_of_every_width(dtype, dk, dv):
    """Two heads in runs, 16 value channels a workgroup."""
    c = make(1, 2, 1, 64 * 42 + 3, dk, dv, dtype, seed=dk + dv)
    out, last, _ = forward(c, on_gpu(c))
    check_forward(c, out, last)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dk", [40, 64, 96, 128, 160])
def test_runs_of_many_heads_of_every_width(dk, dtype):
    """16 heads of 64 value channels in six runs of eight chunks: both passes take 32 channels a workgroup, the first one the columns of
    the identity too."""
    B, H, N, dv = 1, 16, 64 * 48 - 7, 64
    c = make(B, H, H, N, dk, dv, dtype, seed=dk)
    out, last, _ = forward(c, on_gpu(c))
    ref, s = np.zeros((B, H, N, dv)), np.array(c["state"])
    for t in range(N):   # (all heads at once; the states of all tokens would be gigabytes)
        key, qry = c["k"][:, :, t], c["q"][:, :, t]
        s *= np.exp(c["g"][:, :, t])[..., None, None]
        u = c["beta"][:, :, t, None] * (c["v"][:, :, t] - np.matmul(key[:, :, None], s)[:, :, 0])
        s += key[..., None] * u[:, :, None]
        ref[:, :, t] = c["scale"] * np.matmul(qry[:, :, None], s)[:, :, 0]
    check(out, ref, dtype, chain(c), "out")
    check(last, s, "f32", chain(c), "state")


def test_a_captured_single_token_replayed():
    """The state in place from replay to replay, on views of one projection; the bits of calls one after the other."""
    B, H, Hk, dk, dv, T = 3, 4, 2, 40, 24, 5
    c = make(B, H, Hk, T, dk, dv, "bf16", seed=23)
    g = on_gpu(c)
    widths = (Hk * dk, Hk * dk, H * dv)
    cat = lambda t: torch.cat([g[n][:, :, t].reshape(B, -1) for n in ("q", "k", "v")], -1)
    one, scalars = cat(0), torch.stack((g["g"][:, :, 0], g["beta"][:, :, 0]), 1)
    q, k, v = (p.unflatten(-1, (-1, w)) for p, w in zip(one.split(widths, -1), (dk, dk, dv)))
    state, out = g["state"].clone(), torch.empty((B, H, dv), dtype=torch.bfloat16, device="cuda")
    step = lambda: lf.linfusion_delta_step(q, k, v, scalars[:, 0], scalars[:, 1], state, state, out, scale=c["scale"])
    outs = torch.empty_like(g["v"])

    def feed(t):
        one.copy_(cat(t))
        scalars.copy_(torch.stack((g["g"][:, :, t], g["beta"][:, :, t]), 1))

    for t in range(T):
        feed(t)
        step()
        outs[:, :, t] = out
    check_forward(c, outs, state)
    last = state.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state.copy_(g["state"])
    for t in range(T):
        feed(t)
        out.fill_(float("nan"))
        torch.randn(1 << 18, device="cuda").sum()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, outs[:, :, t])
    assert torch.equal(state, last)

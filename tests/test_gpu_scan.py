"""The gated linear recurrence on the GPU against fp64: sequences, gradients, single tokens."""
import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import layers_oracle as orc
from tests.layers_parity import CODE, STEPS, TORCH, columns, f64, half_step, live, near, stored, within  # noqa: F401

pytestmark = pytest.mark.gpu

FLAGS = {"norm": 0, "leaky": lf.FLAG_SCAN_LEAKY, "sum": lf.FLAG_SCAN_SUM}


def make(B, N, C, dtype, seed, weight="norm", inputs=True, state=True, reverse=False, lengths=None):
    r = np.random.RandomState(seed)
    clip = lambda x: np.clip(x, -6.0, 6.0)
    c = {"dims": (B, N, C), "dtype": dtype, "weight": weight, "reverse": reverse, "lengths": lengths, "t": {}, "w": {}}
    wide = {"x": r.randn(B, N, C), "gate": clip(r.randn(B, N, C)), "input": clip(r.randn(B, N, C)) if inputs else None,
            "dout": r.randn(B, N, C)}
    for n, x in wide.items():
        c["t"][n], c["w"][n] = (None, None) if x is None else stored(x, dtype)
    c["t"]["rate"], c["w"]["rate"] = stored(np.exp(r.uniform(-4, 1.5, C)), "f32")
    for n in ("state_in", "dstate_out"):
        c["t"][n], c["w"][n] = stored(r.randn(B, C), "f32") if state else (None, None)
    return c


def on_gpu(c, spoil=True):
    """The inputs on the GPU; what lies behind a row's length is NaN."""
    g = {n: None if t is None else t.cuda() for n, t in c["t"].items()}
    g["lengths"] = None if c["lengths"] is None else torch.tensor(c["lengths"], dtype=torch.int32, device="cuda")
    if c["lengths"] is not None and spoil:
        dead = torch.from_numpy(~live(c["dims"], c["lengths"])).cuda()
        for n in ("x", "gate", "input", "dout"):
            if g[n] is not None:
                g[n][dead] = float("nan")
    return g


def flags(c):
    return FLAGS[c["weight"]] | (lf.FLAG_SCAN_REVERSE if c["reverse"] else 0)


def memory(size):
    return torch.full((max(16, size),), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read before it is written)


def forward(c, g, saved=True):
    out = torch.full_like(g["x"], 7.0, memory_format=torch.contiguous_format)
    last = torch.full(c["dims"][::2], float("nan"), device="cuda")
    keep = memory(lf.linfusion_scan_saved_bytes(*c["dims"])) if saved else None
    lf.linfusion_scan_fwd(g["x"], g["gate"], g["input"], g["rate"], out, state_in=g["state_in"], state_out=last, saved=keep,
                          lengths=g["lengths"], flags=flags(c), workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
    return out, last, keep


def backward(c, g, keep):
    d = {"d" + n: torch.full_like(g[n], 7.0, memory_format=torch.contiguous_format) for n in ("x", "gate", "input", "rate") if g[n] is not None}
    d.setdefault("dinput", None)
    d["dstate_in"] = torch.full(c["dims"][::2], float("nan"), device="cuda")
    size = lf.linfusion_scan_bwd_workspace_bytes(*c["dims"]) - (0 if keep is None else lf.linfusion_scan_saved_bytes(*c["dims"]))
    lf.linfusion_scan_bwd(g["x"], g["gate"], g["input"], g["rate"], g["dout"], d["dx"], d["dgate"], d["dinput"], d["drate"],
                          state_in=g["state_in"], dstate_out=g["dstate_out"], dstate_in=d["dstate_in"], saved=keep, lengths=g["lengths"],
                          flags=flags(c), workspace=memory(size))
    return {n: t for n, t in d.items() if t is not None}


def reference(c):
    w = c["w"]
    out, last, held = orc.scan(w["x"], w["gate"], w["input"], w["rate"], w["state_in"], c["weight"], c["reverse"], c["lengths"])
    g, e = orc.scan_gradients(w["x"], w["input"], w["rate"], held, w["dout"], w["dstate_out"], c["reverse"], c["lengths"])
    return out, last, held, g, e


def check_all(c, out, last, grads, what=""):
    ref, ref_last, held, g, e = reference(c)
    dtype, on = c["dtype"], live(c["dims"], c["lengths"])
    n = STEPS[dtype]
    near(f64(out)[on], ref[on], dtype, n, held["scale"][on], what + "out")
    assert bool((out[torch.from_numpy(~on).cuda()] == 7.0).all()), what + "out behind a row's length"
    near(last, ref_last, "f32", n, held["last_scale"], what + "state_out")
    for name, got in (grads or {}).items():
        if name in ("drate", "dstate_in"):   # sums over B * N terms: a thread's, a chunk's 32, and fp64
            near(got, g[name], "f32", 2 * n + 8 + (40 if name == "drate" else 0), e[name], what + name)
        else:
            near(f64(got)[on], g[name][on], dtype, 2 * n + 8, e[name][on], what + name)
            assert bool((got[torch.from_numpy(~on).cuda()] == 7.0).all()), what + name + " behind a row's length"


SHAPES = [(1, 1, 8), (2, 2, 8), (1, 3, 72), (2, 37, 64), (3, 127, 40), (1, 128, 16), (2, 129, 136), (1, 255, 8), (1, 256, 64), (1, 257, 24),
          (2, 640, 72), (1, 1025, 200), (1, 5003, 8), (4, 300, 320)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight,inputs,state,reverse", [("norm", True, True, False), ("norm", False, False, True), ("leaky", True, False, True),
                                                         ("leaky", False, True, False), ("sum", True, True, True), ("sum", False, False, False)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_the_oracle(shape, weight, inputs, state, reverse, dtype):
    c = make(*shape, dtype, sum(shape), weight, inputs, state, reverse)
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    check_all(c, out, last, grads)
    again = backward(c, g, None)   # without what the forward pass saved: the same
    assert all(torch.equal(grads[n], again[n]) for n in grads)
    plain = forward(c, g, saved=False)
    assert torch.equal(plain[0], out) and torch.equal(plain[1], last)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight,inputs,state,reverse,ragged", [("norm", True, True, False, False), ("norm", True, True, True, True), ("leaky", False, False, True, False),
                                                                ("sum", True, True, False, True)])
@pytest.mark.parametrize("shape", [(5, 1, 72), (33, 2, 8), (7, 4, 64), (70, 5, 40), (65, 8, 136), (33, 13, 136), (6, 16, 8), (17, 17, 72), (11, 32, 200)], ids=str)
def test_many_rows_of_a_few_tokens(shape, weight, inputs, state, reverse, ragged, dtype):
    """Several rows share a workgroup; the last one has some to spare."""
    B, N, C = shape
    c = make(B, N, C, dtype, sum(shape), weight, inputs, state, reverse, tuple((5 * b + 3) % (N + 1) for b in range(B)) if ragged else None)
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    check_all(c, out, last, grads)
    again = backward(c, g, None)
    assert all(torch.equal(grads[n], again[n]) for n in grads)
    if state:
        held, slope = g["state_in"].clone(), g["dstate_out"].clone()
        more = {n: torch.full_like(t, 7.0) for n, t in grads.items()}
        lf.linfusion_scan_fwd(g["x"], g["gate"], g["input"], g["rate"], torch.empty_like(out), state_in=held, state_out=held, lengths=g["lengths"],
                              flags=flags(c), workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
        lf.linfusion_scan_bwd(g["x"], g["gate"], g["input"], g["rate"], g["dout"], more["dx"], more["dgate"], more.get("dinput"), more["drate"],
                              state_in=g["state_in"], dstate_out=slope, dstate_in=slope, lengths=g["lengths"], flags=flags(c),
                              workspace=memory(lf.linfusion_scan_bwd_workspace_bytes(*c["dims"])))
        assert torch.equal(held, last) and torch.equal(slope, grads["dstate_in"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("N,lengths", [(300, (300, 0, 1, 129)), (700, (128, 256, 257, 699)), (100, (0, 0, 5, 100)), (1100, (-3, 2000, 1024, 513))], ids=str)
def test_ragged_rows(N, lengths, reverse, dtype):
    c = make(4, N, 72, dtype, N, reverse=reverse, lengths=lengths)
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    check_all(c, out, last, backward(c, g, keep))
    if 0 in lengths:
        at = lengths.index(0)
        assert torch.equal(last[at], g["state_in"][at])


@pytest.mark.parametrize("dtype,reverse", [("f32", False), ("bf16", True)])
def test_long_rows_of_few_channels(dtype, reverse):
    """Hundreds of chunks with few beside them: more than a stretch of groups, and exactly one; the same from run to run, states in place."""
    c = make(2, 40000, 72, dtype, 12, reverse=reverse, lengths=(40000, 32768))
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    check_all(c, out, last, grads)
    for _ in range(3):
        again, state = torch.full_like(out, 7.0), g["state_in"].clone()
        lf.linfusion_scan_fwd(g["x"], g["gate"], g["input"], g["rate"], again, state_in=state, state_out=state, lengths=g["lengths"],
                              flags=flags(c), workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
        assert torch.equal(again, out) and torch.equal(state, last)
        more = backward(c, g, None)
        assert all(torch.equal(grads[n], more[n]) for n in grads)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_columns_of_one_buffer(dtype):
    c = make(2, 400, 72, dtype, 5)
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    v = dict(g)
    v["x"], v["gate"], v["input"], v["dout"], out2 = columns([g["x"], g["gate"], g["input"], g["dout"], torch.full_like(out, 7.0)], 8)
    lf.linfusion_scan_fwd(v["x"], v["gate"], v["input"], v["rate"], out2, state_in=g["state_in"], flags=flags(c),
                          workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
    assert torch.equal(out2, out)
    d = columns([torch.full_like(out, 7.0)] * 3)
    lf.linfusion_scan_bwd(v["x"], v["gate"], v["input"], v["rate"], v["dout"], *d, drate := torch.empty_like(g["rate"]),
                          state_in=g["state_in"], dstate_out=g["dstate_out"], saved=keep, flags=flags(c),
                          workspace=memory(lf.linfusion_scan_bwd_workspace_bytes(*c["dims"])))
    for got, n in zip((*d, drate), ("dx", "dgate", "dinput", "drate")):
        assert torch.equal(got, grads[n]), n
    turned = lambda t: t.permute(1, 0, 2).contiguous().permute(1, 0, 2)   # [N, B, C] tensors
    v = {n: turned(g[n]) if n in ("x", "gate", "input", "dout") else g[n] for n in g}
    lf.linfusion_scan_fwd(v["x"], v["gate"], v["input"], v["rate"], out2 := turned(torch.full_like(out, 7.0)), state_in=g["state_in"],
                          flags=flags(c), workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
    assert torch.equal(out2, out)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_state_in_place_and_a_sequence_in_parts(dtype):
    """A sequence in three calls, the state handed on in place, is near the sequence in one."""
    c = make(2, 900, 64, dtype, 9)
    g = on_gpu(c)
    ref, ref_last, held, _, _ = reference(c)
    state, out = g["state_in"].clone(), torch.empty_like(g["x"])
    for at, end in ((0, 1), (1, 390), (390, 900)):
        part = {n: g[n][:, at:end] for n in ("x", "gate", "input")}
        lf.linfusion_scan_fwd(part["x"], part["gate"], part["input"], g["rate"], out[:, at:end], state_in=state, state_out=state,
                              workspace=memory(lf.linfusion_scan_workspace_bytes(2, end - at, 64)))
    near(out, ref, dtype, STEPS[dtype], held["scale"], "out")
    near(state, ref_last, "f32", STEPS[dtype], held["last_scale"], "state")


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("N", [5, 128, 250, 300, 2300])   # one chunk of either length, two, more than a group of them
def test_states_in_place_are_the_same(N, reverse):
    """Every workgroup and wave that starts from the state that is given reads it before the last one replaces it."""
    c = make(3, N, 1280, "bf16", 16, reverse=reverse, lengths=(N, max(1, N // 2), 0))
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    d = backward(c, g, keep)
    for _ in range(4):
        state, again = g["state_in"].clone(), torch.full_like(out, 7.0)
        lf.linfusion_scan_fwd(g["x"], g["gate"], g["input"], g["rate"], again, state_in=state, state_out=state, lengths=g["lengths"],
                              flags=flags(c), workspace=memory(lf.linfusion_scan_workspace_bytes(*c["dims"])))
        assert torch.equal(again, out) and torch.equal(state, last)
        slope, grads = g["dstate_out"].clone(), {n: torch.full_like(t, 7.0) for n, t in d.items()}
        lf.linfusion_scan_bwd(g["x"], g["gate"], g["input"], g["rate"], g["dout"], grads["dx"], grads["dgate"], grads["dinput"], grads["drate"],
                              state_in=g["state_in"], dstate_out=slope, dstate_in=slope, saved=keep, lengths=g["lengths"], flags=flags(c),
                              workspace=memory(lf.linfusion_scan_bwd_workspace_bytes(*c["dims"])))
        assert torch.equal(slope, d["dstate_in"])
        assert all(torch.equal(grads[n], d[n]) for n in d if n != "dstate_in")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight,inputs", [("norm", True), ("norm", False), ("leaky", True), ("sum", True)])
@pytest.mark.parametrize("B,C", [(1, 8), (3, 40), (64, 520), (2, 4096)])
def test_single_tokens(B, C, weight, inputs, dtype):
    c = make(B, 3, C, dtype, B + C, weight, inputs)
    g = on_gpu(c)
    ref, ref_last, held, _, _ = reference(c)
    state, out = g["state_in"].clone(), torch.full_like(g["x"], float("nan"))
    for t in range(3):
        row = lambda n: None if g[n] is None else g[n][:, t]
        lf.linfusion_scan_step(row("x"), row("gate"), row("input"), g["rate"], state, state, out[:, t], flags=flags(c))
    near(out, ref, dtype, STEPS[dtype], held["scale"], "out")
    near(state, ref_last, "f32", STEPS[dtype], held["last_scale"], "state")
    fresh = torch.empty_like(out[:, 0])
    lf.linfusion_scan_step(row("x"), row("gate"), row("input"), g["rate"], None, None, fresh, flags=flags(c) | lf.FLAG_SCAN_REVERSE)
    w = c["w"]
    one = orc.scan(*(w[n][:, 2:] if w[n] is not None else None for n in ("x", "gate", "input")), w["rate"], None, weight)
    near(fresh, one[0][:, 0], dtype, STEPS[dtype], one[2]["scale"][:, 0], "from nothing")


def test_slow_channels_keep_their_weight():
    """sqrt(1 - a^2) where a is next to 1: the series, not a difference of numbers near 1."""
    c = make(1, 200, 64, "f32", 11)
    r = 10.0 ** np.linspace(-12, 0, 64)
    c["t"]["rate"], c["w"]["rate"] = stored(r, "f32")
    g = on_gpu(c)
    out, last, keep = forward(c, g)
    check_all(c, out, last, backward(c, g, keep))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gates_shut_and_wide_open(dtype):
    """Gates of the type's extremes: a = 1 leaves the state, its weight and its gradients 0; a = e^-rate."""
    c = make(2, 300, 64, dtype, 12)
    most = float(torch.finfo(TORCH[dtype]).max)
    g = on_gpu(c)
    g["gate"][:, 100:200] = -most
    g["gate"][:, 200:210] = most
    g["input"][:, 50:60] = -most
    g["input"][:, 60:70] = most
    for n in ("gate", "input"):
        c["w"][n] = f64(g[n])
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    with np.errstate(over="ignore", invalid="ignore"):
        check_all(c, out, last, grads)   # (equal outputs while the gate is shut only to rounding: a thread's first state is A h + R)
    assert bool((grads["dgate"][:, 100:200] == 0).all()) and bool((grads["dx"][:, 100:200] == 0).all())
    g["rate"].zero_()   # a = 1 everywhere, m = 0
    out, last, keep = forward(c, g)
    grads = backward(c, g, keep)
    assert torch.equal(last, g["state_in"]) and all(bool(torch.isfinite(t).all()) for t in grads.values())


def test_infinities_stay_in_their_channel():
    c = make(1, 600, 64, "f32", 13)
    g = on_gpu(c)
    clean, _, _ = forward(c, g)
    g["x"][0, 300, 5] = float("nan")
    g["x"][0, 400, 9] = float("inf")
    out, _, _ = forward(c, g)
    other = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(out[..., other], clean[..., other])
    assert torch.equal(out[0, :300], clean[0, :300])
    assert bool(torch.isnan(out[0, 300:, 5]).all()) and bool((~torch.isfinite(out[0, 400:, 9])).all())


def test_gradients_against_differences():
    """Directional derivatives of sum(out * dout) + sum(state * dstate) by central differences of the fp64 oracle."""
    c = make(2, 70, 16, "f32", 14, lengths=(70, 33))
    g = on_gpu(c)
    grads = backward(c, g, forward(c, g)[2])
    w, r = c["w"], np.random.RandomState(3)
    on = live(c["dims"], c["lengths"])[..., None]

    def loss(v):
        out, last, _ = orc.scan(v["x"], v["gate"], v["input"], v["rate"], v["state_in"], "norm", False, c["lengths"])
        return (out * w["dout"] * on).sum() + (last * w["dstate_out"]).sum()

    for n in ("x", "gate", "input", "rate", "state_in"):
        d = r.randn(*w[n].shape)
        if n in ("x", "gate", "input"):
            d = d * on
        step = 1e-6
        want = (loss(w | {n: w[n] + step * d}) - loss(w | {n: w[n] - step * d})) / (2 * step)
        got = f64(grads["d" + n])
        got = (np.where(on, got, 0.0) if got.ndim == 3 else got) * d
        # the difference's own error: step^2 of the third derivative and 1e-16 / step of the loss; the gradients': fp32
        assert abs(got.sum() - want) <= 1e-5 * np.abs(got).sum() + 1e-7 * abs(loss(w)), n


def test_graphs_that_share_a_workspace_replayed_beside_eager_calls():
    c = make(2, 700, 72, "bf16", 15)
    g = on_gpu(c)
    want = forward(c, g)
    want_grads = backward(c, g, want[2])
    out, last, keep = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(want[2])
    ws = memory(max(lf.linfusion_scan_workspace_bytes(*c["dims"]), lf.linfusion_scan_bwd_workspace_bytes(*c["dims"])))
    d = {n: torch.empty_like(t) for n, t in want_grads.items()}
    rest = {"state_in": g["state_in"], "saved": keep, "workspace": ws}
    stream = torch.cuda.Stream()
    graphs = []
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for call in (lambda: lf.linfusion_scan_fwd(g["x"], g["gate"], g["input"], g["rate"], out, state_out=last, **rest),
                     lambda: lf.linfusion_scan_bwd(g["x"], g["gate"], g["input"], g["rate"], g["dout"], d["dx"], d["dgate"], d["dinput"], d["drate"],
                                                   dstate_out=g["dstate_out"], dstate_in=d["dstate_in"], **rest)):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                call()
        for _ in range(4):
            ws.fill_(255)
            for t in (out, last, *d.values()):
                t.zero_()
            graphs[0].replay()
            graphs[1].replay()
            stream.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(last, want[1])
            assert all(torch.equal(d[n], want_grads[n]) for n in d)
            assert torch.equal(forward(c, g)[0], want[0])


def test_two_calls_at_once_with_workspaces_of_their_own():
    cases = [make(1, 3000, 64, "bf16", 16), make(2, 2000, 128, "f32", 17)]
    gs = [on_gpu(c) for c in cases]
    want = [forward(c, g) for c, g in zip(cases, gs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(forward(cases[i], gs[i])[:2])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i][0]) and torch.equal(l, want[i][1]) for o, l in got[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_stream(dtype):
    """Hundreds of chunks against the recurrence in fp64 on the GPU."""
    B, N, C = 1, 40000, 128
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, gate, inp = (torch.randn((B, N, C), generator=gen, device="cuda").clamp(-6, 6).to(TORCH[dtype]) for _ in range(3))
    rate = torch.exp(torch.rand(C, generator=gen, device="cuda") * 8 - 7)
    out, last = torch.empty_like(x), torch.empty((B, C), device="cuda")
    lf.linfusion_scan_fwd(x, gate, inp, rate, out, state_out=last, workspace=memory(lf.linfusion_scan_workspace_bytes(B, N, C)))
    s = torch.sigmoid(gate.double())
    decay = rate.double() * s
    a, u = torch.exp(-decay), torch.sqrt(-torch.expm1(-2 * decay)) * torch.sigmoid(inp.double()) * x.double()
    h, e = torch.zeros((B, C), dtype=torch.float64, device="cuda"), torch.zeros((B, C), dtype=torch.float64, device="cuda")
    ref, scale = torch.empty_like(u), torch.empty_like(u)
    for t in range(N):
        e = a[:, t] * e + (1 + decay[:, t]) * a[:, t] * h.abs() + u[:, t].abs()
        h = a[:, t] * h + u[:, t]
        ref[:, t], scale[:, t] = h, e
    near(out, f64(ref), dtype, STEPS[dtype], f64(scale), "out")
    near(last, f64(h), "f32", STEPS[dtype], f64(e), "state")


def test_rows_beyond_4_gib():
    """A view whose token stride puts its last rows more than 2^32 bytes behind its first."""
    B, N, C = 1, 300, 8
    wide = torch.zeros((N, 1 << 23), dtype=torch.bfloat16, device="cuda")   # 16 MiB a row, 4.7 GiB
    x, gate = wide[:, :C].unsqueeze(0), wide[:, 64:64 + C].unsqueeze(0)
    gen = torch.Generator(device="cuda").manual_seed(6)
    x.copy_(torch.randn((B, N, C), generator=gen, device="cuda"))
    gate.copy_(torch.randn((B, N, C), generator=gen, device="cuda"))
    rate = torch.ones(C, device="cuda")
    got, want = wide[:, 128:128 + C].unsqueeze(0), torch.empty((B, N, C), dtype=torch.bfloat16, device="cuda")
    ws = memory(lf.linfusion_scan_workspace_bytes(B, N, C))
    lf.linfusion_scan_fwd(x, gate, None, rate, got, workspace=ws)
    lf.linfusion_scan_fwd(x.contiguous(), gate.contiguous(), None, rate, want, workspace=ws)
    assert torch.equal(got.contiguous(), want)

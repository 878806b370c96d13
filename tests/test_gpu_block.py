"""Whole blocks as a user builds them: boundary, projections, positions, mixer, boundary; forward and gradients in fp32, forward
in 16 bits, and tokens one at a time behind a prompt.  The projections are torch's products, on both sides."""
import numpy as np
import pytest
import torch

import paper_2409_02097_amd as lf
from oracle import block_oracle as orc
from oracle import linattn_oracle
from tests.block_parity import TORCH, check, f64

pytestmark = pytest.mark.gpu

B, N, H, HK, D, DV = 2, 96, 4, 2, 32, 48
C = 128
GRID = (12, 8)
CHANNELS, BASES, EPS = (16, 16), (1e4, 1e4), 1e-6


def weights(seed):
    r = np.random.RandomState(seed)
    mat = lambda a, b: r.randn(a, b) / np.sqrt(a)
    return {"x": r.randn(B, N, C), "scale": 0.2 * r.randn(B, C), "shift": 0.2 * r.randn(B, C), "gate": 0.5 * r.randn(B, C),
            "scale2": 0.2 * r.randn(B, C), "shift2": 0.2 * r.randn(B, C), "wq": mat(C, HK * D), "wk": mat(C, HK * D), "wv": mat(C, H * DV),
            "wo": mat(H * DV, C), "g": -np.exp(r.uniform(-6, 0, (B, H, N))), "beta": r.uniform(0, 1, (B, H, N)),
            "dy": r.randn(B, N, C), "dh": r.randn(B, N, C)}


def positions():
    n = torch.arange(N)
    return torch.stack([n // GRID[1], n % GRID[1]]).int()


def exact(w):
    """The block and its gradients with respect to x and the vectors, fp64 torch on the CPU, the recurrence token by token."""
    t = {n: torch.from_numpy(v).double().requires_grad_(n not in ("dy", "dh")) for n, v in w.items()}

    def unit(v):
        v = v - v.mean(-1, keepdim=True)
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)

    def turn(v):
        at, parts = 0, []
        for a, c in enumerate(CHANNELS):
            theta = positions()[a].double()[:, None] * BASES[a] ** (-2.0 * torch.arange(c // 2, dtype=torch.float64) / c)
            one, two = v[..., at:at + c // 2], v[..., at + c // 2:at + c]
            parts += [one * torch.cos(theta) - two * torch.sin(theta), two * torch.cos(theta) + one * torch.sin(theta)]
            at += c
        return torch.cat(parts, -1)

    h = unit(t["x"]) * (1 + t["scale"][:, None]) + t["shift"][:, None]
    heads = lambda v, n, d: v.view(B, N, n, d).permute(0, 2, 1, 3)
    q, k, v = heads(h @ t["wq"], HK, D), heads(h @ t["wk"], HK, D), heads(h @ t["wv"], H, DV)
    q, k = (turn(torch.nn.functional.normalize(m, dim=-1)).repeat_interleave(H // HK, 1) for m in (q, k))
    s, out = torch.zeros(B, H, D, DV, dtype=torch.float64), []
    for i in range(N):
        s = s * torch.exp(t["g"][:, :, i])[..., None, None]
        u = t["beta"][:, :, i, None] * (v[:, :, i] - (k[:, :, i, None] @ s)[..., 0, :])
        s = s + k[:, :, i, :, None] * u[..., None, :]
        out.append(D ** -0.5 * (q[:, :, i, None] @ s)[..., 0, :])
    f = torch.stack(out, 2).permute(0, 2, 1, 3).reshape(B, N, H * DV) @ t["wo"]
    y = t["x"] + t["gate"][:, None] * f
    h2 = unit(y) * (1 + t["scale2"][:, None]) + t["shift2"][:, None]
    ((y * t["dy"]).sum() + (h2 * t["dh"]).sum()).backward()
    return y.detach().numpy(), h2.detach().numpy(), {n: v.grad.numpy() for n, v in t.items() if v.grad is not None}, s.detach().numpy()


def heads(v, n, d):
    return v.view(B, -1, n, d).permute(0, 2, 1, 3)


def run(w, dtype, backward):
    """The same with the framework's operators; gradients by its own backward calls."""
    T = TORCH[dtype]
    t = {n: torch.from_numpy(v).cuda().to(torch.float32 if n in ("scale", "shift", "gate", "scale2", "shift2", "g", "beta") else T)
         for n, v in w.items()}
    pos, code = positions().cuda(), {"f32": 0, "f16": 1, "bf16": 2}[dtype]
    h = torch.empty_like(t["x"])
    lf.linfusion_gate_norm_fwd(t["x"], None, None, t["scale"], t["shift"], None, h)
    raw = {n: heads(h @ t["w" + n], HK, D) for n in ("q", "k")}
    unit = {n: torch.nn.functional.normalize(x.float(), dim=-1).to(T) for n, x in raw.items()}
    v = heads(h @ t["wv"], H, DV)
    q, k = (torch.empty_like(unit[n]) for n in ("q", "k"))
    lf.linfusion_rope(unit["q"], unit["k"], q, k, pos, CHANNELS, BASES)
    o = torch.empty((B, N, H, DV), dtype=T, device="cuda").permute(0, 2, 1, 3)
    state = torch.empty((B, H, D, DV), device="cuda")
    saved = torch.empty(lf.linfusion_delta_saved_bytes(B, H, HK, N, D, DV, code), dtype=torch.uint8, device="cuda")
    lf.linfusion_delta_fwd(q, k, v, t["g"], t["beta"], o, scale=D ** -0.5, state_out=state, saved=saved)
    flat = o.permute(0, 2, 1, 3).reshape(B, N, H * DV)
    f = flat @ t["wo"]
    y, h2 = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    lf.linfusion_gate_norm_fwd(t["x"], f, t["gate"], t["scale2"], t["shift2"], y, h2)
    if not backward:
        return y, h2, None, state
    grads = {n: torch.empty_like(t[n]) for n in ("gate", "scale", "shift", "scale2", "shift2")}
    ws = torch.empty(lf.linfusion_gate_norm_bwd_workspace_bytes(B, N, C), dtype=torch.uint8, device="cuda")
    dx, df = torch.empty_like(y), torch.empty_like(y)
    lf.linfusion_gate_norm_bwd(t["x"], f, t["gate"], t["scale2"], t["dy"], t["dh"], dx, df, grads["gate"], grads["scale2"], grads["shift2"],
                               workspace=ws)
    grads["wo"] = flat.view(-1, H * DV).t() @ df.view(-1, C)
    do = heads(df @ t["wo"].t(), H, DV)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    grads["g"], grads["beta"] = torch.empty_like(t["g"]), torch.empty_like(t["beta"])
    dws = torch.empty(lf.linfusion_delta_bwd_workspace_bytes(B, H, HK, N, D, DV, code), dtype=torch.uint8, device="cuda")
    lf.linfusion_delta_bwd(q, k, v, t["g"], t["beta"], do, dq, dk, dv, grads["g"], grads["beta"], scale=D ** -0.5, saved=saved, workspace=dws)
    lf.linfusion_rope(dq, dk, dq, dk, pos, CHANNELS, BASES, flags=lf.FLAG_ROPE_INVERSE)
    dh = torch.zeros_like(h)
    for n, d in (("q", dq), ("k", dk)):
        x = raw[n].detach().requires_grad_()
        d = torch.autograd.grad(torch.nn.functional.normalize(x, dim=-1), x, d)[0].permute(0, 2, 1, 3).reshape(B, N, HK * D)
        grads["w" + n] = h.view(-1, C).t() @ d.reshape(-1, HK * D)
        dh += d @ t["w" + n].t()
    d = dv.permute(0, 2, 1, 3).reshape(B, N, H * DV)
    grads["wv"] = h.view(-1, C).t() @ d.reshape(-1, H * DV)
    dh += d @ t["wv"].t()
    lf.linfusion_gate_norm_bwd(t["x"], None, None, t["scale"], dx, dh, dx, None, None, grads["scale"], grads["shift"], workspace=ws)
    grads["x"] = dx
    return y, h2, grads, state


# A product over C, H DV or B N terms, the delta rule's chain, four norms' sums: lengths added up, times 4 for the factors
# (rates, 1 + scale, projections) by which one stage's error enters the next.
CHAIN = 4 * (3 * (64 + D + DV) + 3 * C + H * DV + 4 * 48)


def test_block_in_fp32_with_gradients():
    w = {n: v.astype(np.float32).astype(np.float64) for n, v in weights(3).items()}
    ry, rh, rg, rs = exact(w)
    y, h, grads, state = run(w, "f32", True)
    check(y, ry, "f32", CHAIN, "y")
    check(h, rh, "f32", CHAIN, "h")
    check(state, rs, "f32", CHAIN, "state")
    assert set(grads) == set(rg)
    for n, g in grads.items():   # (a sum over B N tokens more for weights and vectors; dg and dbeta sum terms that cancel)
        extra = 64 if n in ("g", "beta") else 1
        check(g, rg[n], "f32", CHAIN + B * N, "d" + n, scale=extra * np.abs(rg[n]).max())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_block_in_16_bits(dtype):
    w = weights(4)
    for n in ("x", "wq", "wk", "wv", "wo"):
        w[n] = torch.from_numpy(w[n]).to(TORCH[dtype]).double().numpy()
    for n in ("scale", "shift", "gate", "scale2", "shift2", "g", "beta"):
        w[n] = w[n].astype(np.float32).astype(np.float64)
    ry, rh, _, _ = exact(w)
    y, h, _, _ = run(w, dtype, False)
    # each of the nine stages rounds its results by half a step; the stages' gains (rates and projections near 1, 1 + scale and
    # gates below 2) multiply to less than 4, and the roundings of C terms add up like sqrt(C) against results that do too
    half = torch.finfo(TORCH[dtype]).eps / 2
    for got, ref, name in ((y, ry, "y"), (h, rh, "h")):
        assert np.abs(f64(got) - ref).max() <= 9 * 4 * half * np.abs(ref).max(), name


def test_tokens_one_at_a_time_behind_a_prompt():
    """A prompt through the sequence call, then tokens through the single-token call with the prompt's state: the outputs of the
    whole sequence at once."""
    r = np.random.RandomState(6)
    q, k = (torch.nn.functional.normalize(torch.from_numpy(r.randn(B, HK, N, D)).float(), dim=-1).cuda() for _ in range(2))
    v = torch.from_numpy(r.randn(B, H, N, DV)).float().cuda()
    g, beta = torch.from_numpy(-np.exp(r.uniform(-6, 0, (B, H, N)))).float().cuda(), torch.rand(B, H, N, device="cuda")
    pos = positions().cuda()
    tq, tk = torch.empty_like(q), torch.empty_like(k)
    lf.linfusion_rope(q, k, tq, tk, pos, CHANNELS, BASES)
    cut = 70
    out, state = torch.empty_like(v), torch.empty(B, H, D, DV, device="cuda")
    ws = torch.empty(lf.linfusion_delta_workspace_bytes(B, H, HK, N, D, DV, 0), dtype=torch.uint8, device="cuda")
    lf.linfusion_delta_fwd(*(t[:, :, :cut] for t in (tq, tk, v, g, beta)), out[:, :, :cut], state_out=state, workspace=ws)
    for i in range(cut, N):
        qi, ki = (t[:, :, i:i + 1].contiguous() for t in (q, k))
        lf.linfusion_rope(qi, ki, qi, ki, pos[:, i:i + 1].contiguous(), CHANNELS, BASES)
        assert torch.equal(qi, tq[:, :, i:i + 1]) and torch.equal(ki, tk[:, :, i:i + 1])
        lf.linfusion_delta_step(qi[:, :, 0], ki[:, :, 0], v[:, :, i], g[:, :, i], beta[:, :, i], state, state, out[:, :, i])
    wide = [f64(t) for t in (tq, tk, v, g, beta)]
    ref, last, _ = orc.delta(*wide, 1.0)
    check(out, ref, "f32", 3 * (64 + D + DV), "out")
    check(state, last, "f32", 3 * (64 + D + DV), "state")


def test_block_with_the_non_causal_mixer():
    """The boundary and the positions around the linear attention that the framework is built on, on token-major tensors."""
    r = np.random.RandomState(8)
    heads_, d = 8, 40
    x = torch.from_numpy(r.randn(1, 300, heads_ * d)).half().cuda()
    h, y, h2 = (torch.empty_like(x) for _ in range(3))
    scale, shift, gate = (torch.from_numpy(0.3 * r.randn(1, heads_ * d)).float().cuda() for _ in range(3))
    lf.linfusion_gate_norm_fwd(x, None, None, scale, shift, None, h)
    view = lambda t: t.view(1, 300, heads_, d).permute(0, 2, 1, 3)
    pos = torch.stack([torch.arange(300) // 20, torch.arange(300) % 20]).int().cuda()
    q, k, o = (torch.empty_like(h) for _ in range(3))
    lf.linfusion_rope(view(h), view(h), view(q), view(k), pos, (20, 20), (1e4, 1e4))
    ws = torch.empty(lf.linfusion_attn_workspace_bytes(1, heads_, 300, d, lf.DTYPE_F16), dtype=torch.uint8, device="cuda")
    lf.linfusion_attn_fwd_strided(view(q), view(k), view(h), view(o), lf.PHI_ELU_PLUS_ONE, EPS, 0, ws)
    lf.linfusion_gate_norm_fwd(x, o, gate, scale, shift, y, h2)
    hr = orc.boundary(f64(x), None, None, f64(scale), f64(shift), None, None, 1.0, EPS, False, False)[1]
    check(h, hr, "f16", 640, "h")
    turned = orc.rope(f64(view(h)), pos.cpu().numpy(), (20, 20), (1e4, 1e4))
    check(view(q), turned, "f16", 45, "q")
    assert torch.equal(q, k)
    ref = np.stack([linattn_oracle.attention_linear(f64(view(q))[0, i], f64(view(k))[0, i], f64(view(h))[0, i], 0, EPS) for i in range(heads_)])
    assert np.abs(f64(view(o))[0] - ref).max() <= 2e-3 * np.abs(ref).max() + 2.0 ** -11 * np.abs(ref).max()
    ry, rh = orc.boundary(f64(x), f64(o), f64(gate), f64(scale), f64(shift), None, None, 1.0, EPS, False, False)
    check(y, ry, "f16", 8, "y")
    check(h2, rh, "f16", 640, "h2")

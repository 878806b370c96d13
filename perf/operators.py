"""What a transformer block on image or video tokens does around, and in place of, the non-causal token mixer, as cases
that can be timed and compared.

  rope   rotary positions with several axes (height and width, or time, height and width) on the queries and keys of one
         layer.  "inverse" turns them back: the gradient of the forward call.
  norm   the boundary between two blocks: the residual update with its gate, a norm of the block's output before it
         (where "post"), and the modulated norm that the next block starts with.  "train": the gradients too.
  delta  the gated delta rule, a causal linear attention whose state forgets by a gate and corrects what it holds for a
         key: over whole sequences ("fwd"), with its gradients ("train"), and for one new token ("step").

Where `own` is true, run() calls the framework's operators; where it is false, it computes their formulas with elementary
torch operations in 32 bits (angles of positions and sums of log decays in 64).
"""
import math

import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ITEMSIZE = {"f32": 4, "f16": 2, "bf16": 2}
NORM_EPS = 1e-6
BASE = 10000.0
CHUNK = 64


def _rope(name, dtype, B, H, Hk, d, frames, height, width, channels, pairs="half", inverse=False, own_positions=False):
    """`channels`: how many of a head's channels each axis turns, as text: a case holds plain values."""
    return {"name": name, "kind": "rope", "dtype": dtype, "B": B, "H": H, "Hk": Hk, "d": d, "frames": frames,
            "height": height, "width": width, "channels": channels, "pairs": pairs, "inverse": inverse,
            "own_positions": own_positions}


def _norm(name, kind, dtype, B, N, C, rms, post, ragged=False):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "N": N, "C": C, "rms": rms, "post": post,
            "ragged": ragged}


def _delta(name, kind, dtype, B, H, Hk, N, dk, dv, state=False, ragged=False):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "H": H, "Hk": Hk, "N": N, "dk": dk, "dv": dv,
            "state": state, "ragged": ragged}


def listed():
    return [
        # the innermost level of a 512 px image (16 x 16 tokens of 8 x 160 channels), a guidance pair: latency
        _rope("rope_16x16_f16", "f16", 2, 8, 8, 160, 0, 16, 16, "80,80"),
        # a video clip: 13 latent frames of 60 x 104, three axes on heads of 128, neighbouring channels paired
        _rope("rope_video_bf16", "bf16", 1, 16, 16, 128, 13, 60, 104, "32,48,48", pairs="neighbours"),
        # the way back in fp32, on an image of odd size whose heads keep 8 channels without a position
        _rope("rope_211x173_f32_back", "f32", 2, 8, 8, 40, 0, 211, 173, "16,16", inverse=True),
        # the block boundary at the innermost level of a 512 px image: layer norm with modulation, latency
        _norm("norm_256_f16", "norm_fwd", "f16", 2, 256, 1280, False, False),
        # the same on the video clip's tokens, root mean square norms on both sides of the gate
        _norm("norm_video_bf16", "norm_fwd", "bf16", 1, 13 * 60 * 104, 2048, True, True),
        # a training step at 512 px: 96 images over 8 GPUs, 64 x 64 tokens of 320 channels
        _norm("norm_train_4096_bf16", "norm_train", "bf16", 12, 64 * 64, 320, False, False),
        # one new token for one user, and for a batch of 64, whose 16 value heads share 8 query and key heads
        _delta("step_1_bf16", "delta_step", "bf16", 1, 8, 8, 1, 64, 64, state=True),
        _delta("step_64_bf16", "delta_step", "bf16", 64, 16, 8, 1, 128, 128, state=True),
        # a prompt of odd length
        _delta("delta_197_f16", "delta_fwd", "f16", 1, 8, 8, 197, 64, 64),
        # a long stream of few heads: 256 x 256 tokens in raster order
        _delta("delta_65536_bf16", "delta_fwd", "bf16", 1, 10, 10, 256 * 256, 64, 64, state=True),
        # a training step at 512 px, heads of 40
        _delta("delta_train_4096_bf16", "delta_train", "bf16", 12, 8, 8, 64 * 64, 40, 40),
        # one in fp32 on a padded batch of ragged sequences, shared query and key heads, values wider than keys
        _delta("delta_train_ragged_f32", "delta_train", "f32", 3, 8, 4, 1000, 64, 128, state=True, ragged=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "norm_fwd", "norm_train", "delta_step", "delta_fwd", "delta_fwd", "delta_train"))
    dtype = rng.choice(("f16", "bf16", "bf16", "f32"))
    if kind == "rope":
        d, sections = rng.choice(((40, ((20, 20), (16, 16), (40,))), (64, ((32, 32), (16, 24, 24), (64,))),
                                  (80, ((40, 40), (16, 32, 32))), (128, ((64, 64), (32, 48, 48), (44, 42, 42), (128,))),
                                  (160, ((80, 80), (64, 48, 48)))))
        channels = rng.choice(sections)
        H = rng.choice((4, 5, 8, 10, 16))
        Hk = rng.choice((H, H, max(g for g in (1, 2, 4, 5) if H % g == 0)))
        frames = rng.randint(2, 16) if len(channels) == 3 else 0
        most = 160e6 if dtype != "f32" else 80e6
        tokens = _log(rng, 24, max(32.0, most / (H * d)))
        height = max(1, int(math.sqrt(tokens / max(1, frames)) * rng.uniform(0.6, 1.5)))
        width = max(1, tokens // max(1, frames) // height)
        if len(channels) == 1:
            height, width = 1, height * width
        B = rng.choice([b for b in (1, 2, 3, 4) if b * tokens * H * d <= most] or [1])
        case = _rope("", dtype, B, H, Hk, d, frames, height, width, ",".join(map(str, channels)),
                     rng.choice(("half", "neighbours")), rng.random() < 0.4, rng.random() < 0.3)
    elif kind.startswith("norm"):
        C = rng.choice((320, 512, 640, 768, 1152, 1280, 1536, 2048, 2560, 4096, 5120))
        most = 160e6 if kind == "norm_fwd" else 30e6
        B = rng.choice((1, 1, 2, 3, 12))
        case = _norm("", kind, dtype, B, max(1, _log(rng, 1, max(2.0, most / (B * C)))), C, rng.random() < 0.5,
                     rng.random() < 0.5, rng.random() < 0.3)
    else:
        dk = rng.choice((16, 32, 40, 64, 64, 80, 96, 128, 128, 160))
        dv = rng.choice((dk, dk, dk, rng.choice((24, 64, 128))))
        H = rng.choice((2, 4, 5, 8, 8, 10, 16))
        Hk = rng.choice((H, H, H // 2 if H % 2 == 0 else H))
        if kind == "delta_step":
            B = _log(rng, 1, 64)
            return {k: v for k, v in _delta("", kind, dtype, B, H, Hk, 1, dk, dv, state=True).items() if k != "name"}
        most = 40e6 if kind == "delta_fwd" else 15e6
        B = rng.choice((1, 1, 2, 3, 8))
        N = _log(rng, 2, max(64.0, min(40000.0 if kind == "delta_fwd" else 4000.0, most / (B * H * max(dk, dv)))))
        case = _delta("", kind, dtype, B, H, Hk, N, dk, dv, rng.random() < 0.5, rng.random() < 0.4)
    case.pop("name")
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _heads(x):
    """[B, N, H, d] activations as the [B, H, N, d] view that the mixers take."""
    return x.permute(0, 2, 1, 3)


def _lengths(case, gen):
    if not case["ragged"]:
        return None
    n = torch.randint(0, case["N"] + 1, (case["B"],), generator=gen, device="cuda", dtype=torch.int32)
    n[0] = case["N"]
    return n


def _tokens(case):
    return max(1, case["frames"]) * case["height"] * case["width"]


def _prepare_rope(case, gen):
    B, H, Hk, d, dtype = case["B"], case["H"], case["Hk"], case["d"], TORCH_DTYPE[case["dtype"]]
    N = _tokens(case)
    channels = [int(c) for c in case["channels"].split(",")]
    n = torch.arange(N, device="cuda", dtype=torch.int32)
    w, h = case["width"], case["height"]
    axes = {1: (n,), 2: (n // w, n % w), 3: (n // (w * h), n // w % h, n % w)}[len(channels)]
    positions = torch.stack(axes).to(torch.int32)
    if case["own_positions"]:   # each image of the batch at an offset of its own: crops of a larger picture
        at = torch.randint(0, 500, (B, len(channels), 1), generator=gen, device="cuda", dtype=torch.int32)
        positions = positions.unsqueeze(0) + at
    s = {"q": _heads(_normal((B, N, H, d), gen).to(dtype)), "k": _heads(_normal((B, N, Hk, d), gen).to(dtype)),
         "positions": positions.contiguous(), "channels": channels, "neighbours": case["pairs"] == "neighbours",
         "inverse": case["inverse"]}
    for name in ("q", "k"):
        s[name + "_out"] = torch.empty_like(s[name])
    return s


def _prepare_norm(case, gen):
    B, N, C, dtype = case["B"], case["N"], case["C"], TORCH_DTYPE[case["dtype"]]
    train = case["kind"] == "norm_train"
    # a residual stream with a mean of its own, and some channels far larger than the others
    loud = 1.0 + 9.0 * (torch.rand(C, generator=gen, device="cuda") < 0.02)
    s = {"x": (_normal((B, N, C), gen) * loud + 0.3).to(dtype), "f": (_normal((B, N, C), gen) * 0.7).to(dtype),
         "gate": _normal((B, C), gen) * 0.5, "scale": _normal((B, C), gen) * 0.2, "shift": _normal((B, C), gen) * 0.2,
         "w_pre": 1.0 + 0.1 * _normal((C,), gen) if case["rms"] else None,
         "w_post": 1.0 + 0.1 * _normal((C,), gen) if case["post"] else None,
         "rms": case["rms"], "post": case["post"], "lengths": _lengths(case, gen)}
    like = {"y": "x", "h": "x"}
    if train:
        s["dy"], s["dh"] = (_normal((B, N, C), gen).to(dtype) for _ in range(2))
        like |= {"dx": "x", "df": "x", "dgate": "gate", "dscale": "gate", "dshift": "gate"}
        like |= {"d" + w: w for w in ("w_pre", "w_post") if s[w] is not None}
    for name, of in like.items():
        s[name] = torch.zeros_like(s[of])   # what lies behind a row's length stays zero
    return s


def _prepare_delta(case, gen):
    B, H, Hk, N, dk, dv = (case[n] for n in ("B", "H", "Hk", "N", "dk", "dv"))
    dtype = TORCH_DTYPE[case["dtype"]]
    # queries and keys as such layers make them: the positive side of an activation, of unit length
    unit = lambda h: torch.nn.functional.normalize(torch.nn.functional.silu(_normal((B, N, h, dk), gen)), dim=-1)
    s = {"q": _heads(unit(Hk).to(dtype)), "k": _heads(unit(Hk).to(dtype)),
         "v": _heads(_normal((B, N, H, dv), gen).to(dtype))}
    # log decays from 1e-3 to about 1 a token, the slower heads beside the faster ones; corrections between 0 and 1
    rate = torch.exp(torch.rand(H, generator=gen, device="cuda") * 3.0)
    s["g"] = (-rate * torch.nn.functional.softplus(_normal((B, N, H), gen) - 4.0)).permute(0, 2, 1)
    s["beta"] = torch.sigmoid(_normal((B, N, H), gen)).permute(0, 2, 1)
    s["state_in"] = _normal((B, H, dk, dv), gen) * 0.3 if case["state"] else None
    s["out"] = torch.zeros_like(s["v"])
    s["state_out"] = torch.empty((B, H, dk, dv), device="cuda")
    s["q_scale"] = dk ** -0.5
    if case["kind"] == "delta_step":
        for name in ("q", "k", "v", "out"):
            s[name] = s[name][:, :, 0]
        for name in ("g", "beta"):
            s[name] = s[name][:, :, 0]
        return s
    s["lengths"] = _lengths(case, gen)
    if case["kind"] == "delta_train":
        s["dout"] = _heads(_normal((B, N, H, dv), gen).to(dtype))
        s["dstate_out"] = _normal((B, H, dk, dv), gen) * 0.1 if case["state"] else None
        for name in ("q", "k", "v", "g", "beta"):
            s["d" + name] = torch.zeros_like(s[name])
        s["dstate_in"] = torch.empty_like(s["state_out"]) if case["state"] else None
    return s


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    make = _prepare_rope if kind == "rope" else _prepare_norm if kind.startswith("norm") else _prepare_delta
    return dict(make(case, gen), kind=kind)


# ---- the framework's operators --------------------------------------------------------------------------------------


def _kept(s, name, size):
    """A workspace that the program keeps beside its buffers."""
    if name not in s:
        s[name] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return s[name]


def _own_rope(s):
    import paper_2409_02097_amd as lf
    flags = (lf.FLAG_ROPE_NEIGHBOURS if s["neighbours"] else 0) | (lf.FLAG_ROPE_INVERSE if s["inverse"] else 0)
    lf.linfusion_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], s["channels"],
                      [BASE] * len(s["channels"]), flags=flags)
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_norm(s):
    import paper_2409_02097_amd as lf
    flags = (lf.FLAG_NORM_RMS if s["rms"] else 0) | (lf.FLAG_NORM_POST if s["post"] else 0)
    rest = {"w_pre": s["w_pre"], "w_post": s["w_post"], "norm_eps": NORM_EPS, "flags": flags, "lengths": s["lengths"]}
    lf.linfusion_gate_norm_fwd(s["x"], s["f"], s["gate"], s["scale"], s["shift"], s["y"], s["h"], **rest)
    got = {"y": s["y"], "h": s["h"]}
    if s["kind"] == "norm_train":
        B, N, C = s["x"].shape
        ws = _kept(s, "workspace", lambda: lf.linfusion_gate_norm_bwd_workspace_bytes(B, N, C))
        grads = {n: s[n] for n in ("dx", "df", "dgate", "dscale", "dshift", "dw_pre", "dw_post") if n in s}
        lf.linfusion_gate_norm_bwd(s["x"], s["f"], s["gate"], s["scale"], s["dy"], s["dh"], **grads, workspace=ws, **rest)
        got |= grads
    return got


def _own_delta(s):
    import paper_2409_02097_amd as lf
    if s["kind"] == "delta_step":
        lf.linfusion_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state_in"], s["state_out"], s["out"],
                                scale=s["q_scale"])
        return {"out": s["out"], "state": s["state_out"]}
    B, H, N, dv = s["v"].shape
    Hk, dk = s["q"].shape[1], s["q"].shape[3]
    code = {torch.float32: lf.DTYPE_F32, torch.float16: lf.DTYPE_F16, torch.bfloat16: lf.DTYPE_BF16}[s["q"].dtype]
    ws = _kept(s, "workspace", lambda: lf.linfusion_delta_workspace_bytes(B, H, Hk, N, dk, dv, code))
    train = s["kind"] == "delta_train"
    saved = _kept(s, "saved", lambda: lf.linfusion_delta_saved_bytes(B, H, Hk, N, dk, dv, code)) if train else None
    rest = {"scale": s["q_scale"], "state_in": s["state_in"], "lengths": s["lengths"], "saved": saved}
    lf.linfusion_delta_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["out"], state_out=s["state_out"], workspace=ws,
                           **rest)
    got = {"out": s["out"], "state": s["state_out"]}
    if train:
        ws = _kept(s, "bwd_workspace", lambda: lf.linfusion_delta_bwd_workspace_bytes(B, H, Hk, N, dk, dv, code))
        grads = [s[n] for n in ("dq", "dk", "dv", "dg", "dbeta")]
        lf.linfusion_delta_bwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["dout"], *grads,
                               dstate_out=s["dstate_out"], dstate_in=s["dstate_in"], workspace=ws, **rest)
        got |= {n: s[n] for n in ("dq", "dk", "dv", "dg", "dbeta")}
        if s["dstate_in"] is not None:
            got["dstate"] = s["dstate_in"]
    return got


# ---- the plain forms ------------------------------------------------------------------------------------------------


def _plain_rope(s):
    positions = s["positions"] if s["positions"].dim() == 3 else s["positions"].unsqueeze(0)
    turned = []
    for x in (s["q"], s["k"]):
        y, at = x.float(), 0
        parts = []
        for axis, c in enumerate(s["channels"]):
            rate = BASE ** (-2.0 * torch.arange(c // 2, device="cuda", dtype=torch.float64) / c)
            angle = (positions[:, axis].double().unsqueeze(-1) * rate).unsqueeze(1)
            cos, sin = torch.cos(angle).float(), torch.sin(angle).float() * (-1.0 if s["inverse"] else 1.0)
            z = y[..., at:at + c]
            a, b = (z[..., 0::2], z[..., 1::2]) if s["neighbours"] else (z[..., :c // 2], z[..., c // 2:])
            one, two = a * cos - b * sin, b * cos + a * sin
            parts.append(torch.stack((one, two), -1).flatten(-2) if s["neighbours"] else torch.cat((one, two), -1))
            at += c
        parts.append(y[..., at:])
        turned.append(torch.cat(parts, -1).to(x.dtype))
    return {"q": turned[0], "k": turned[1]}


def _normed(x, rms):
    if not rms:
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + NORM_EPS)


def _behind(lengths, x):
    """Which tokens of x, [B, N, ...], lie behind their row's length."""
    n = torch.arange(x.shape[1], device="cuda").view(1, -1) >= lengths.view(-1, 1)
    return n.view(n.shape + (1,) * (x.dim() - 2))


def _plain_boundary(s, x, f, gate, scale, shift, w_pre, w_post):
    if s["post"]:
        f = _normed(f, s["rms"]) * w_post
    y = x + gate.unsqueeze(1) * f
    h = _normed(y, s["rms"])
    if w_pre is not None:
        h = h * w_pre
    return y, h * (1.0 + scale.unsqueeze(1)) + shift.unsqueeze(1)


def _plain_norm(s):
    names = [n for n in ("x", "f", "gate", "scale", "shift", "w_pre", "w_post") if s[n] is not None]
    train = s["kind"] == "norm_train"
    leaves = {n: s[n].detach().float().requires_grad_(train) for n in names}
    y, h = _plain_boundary(s, *(leaves.get(n) for n in ("x", "f", "gate", "scale", "shift", "w_pre", "w_post")))
    none = None if s["lengths"] is None else _behind(s["lengths"], y)
    if none is not None:
        y, h = y.masked_fill(none, 0.0), h.masked_fill(none, 0.0)
    got = {"y": y.detach().to(s["x"].dtype), "h": h.detach().to(s["x"].dtype)}
    if train:
        grads = torch.autograd.grad((y, h), list(leaves.values()), (s["dy"].float(), s["dh"].float()))
        got |= {"d" + n: t.to(s[n].dtype) for n, t in zip(names, grads)}
    return got


def _inverse(a):
    """(I + a)^-1 of strictly lower triangular matrices of CHUNK rows: the inverses of the blocks on the diagonal, two
    of them joined into one of twice the size until there is one."""
    eye = torch.eye(CHUNK, device=a.device, dtype=a.dtype)
    inv, size = eye.expand_as(a), 1
    blocks = torch.arange(CHUNK, device=a.device)
    while size < CHUNK:
        row, col = (blocks // size).view(-1, 1), (blocks // size).view(1, -1)
        below = (row == col + 1) & (col % 2 == 0)
        inv = inv - inv @ (a * below) @ inv
        size *= 2
    return inv


def _chunked(x):
    """[B, H, N, ...] -> [B, H, N / CHUNK, CHUNK, ...], zeros behind the last token."""
    more = -x.shape[2] % CHUNK
    if more:
        x = torch.cat((x, x.new_zeros((x.shape[0], x.shape[1], more) + x.shape[3:])), 2)
    return x.view(x.shape[0], x.shape[1], -1, CHUNK, *x.shape[3:])


def _plain_rule(q, k, v, g, beta, scale, state, none):
    """The gated delta rule by chunks; returns the outputs and the last state."""
    B, H, N, dv = v.shape
    if none is not None:   # what stands behind a row's length changes nothing
        q, k, v = (t.masked_fill(none.unsqueeze(-1), 0.0) for t in (q, k, v))
        g, beta = (t.masked_fill(none, 0.0) for t in (g, beta))
    if k.shape[1] != H:
        q, k = (t.repeat_interleave(H // t.shape[1], 1) for t in (q, k))
    q, k, v, g, beta = (_chunked(t) for t in (q * scale, k, v, g, beta))
    at = g.double().cumsum(-1)
    earlier = torch.ones(CHUNK, CHUNK, device=q.device).tril() > 0
    decay = torch.exp((at.unsqueeze(-1) - at.unsqueeze(-2)).masked_fill(~earlier, -math.inf)).float()
    since, left, whole = torch.exp(at).float(), torch.exp(at[..., -1:] - at).float(), torch.exp(at[..., -1]).float()
    solve = _inverse(((k @ k.transpose(-1, -2)) * decay * beta.unsqueeze(-1)).tril(-1))
    w = (solve @ (k * (beta * since).unsqueeze(-1))).unbind(2)
    u = (solve @ (v * beta.unsqueeze(-1))).unbind(2)
    within = ((q @ k.transpose(-1, -2)) * decay).unbind(2)
    read, write = (q * since.unsqueeze(-1)).unbind(2), (k * left.unsqueeze(-1)).transpose(-1, -2).unbind(2)
    whole = whole.unsqueeze(-1).unsqueeze(-1).unbind(2)
    out = []
    for i in range(len(u)):
        new = u[i] - w[i] @ state
        out.append(read[i] @ state + within[i] @ new)
        state = whole[i] * state + write[i] @ new
    return torch.cat(out, 2)[:, :, :N], state


def _plain_delta(s):
    state = s["state_in"]
    if state is None:
        state = torch.zeros_like(s["state_out"])
    if s["kind"] == "delta_step":
        q, k, v = (s[n].float() for n in ("q", "k", "v"))
        q, k = (t.repeat_interleave(v.shape[1] // t.shape[1], 1) for t in (q, k))
        state = state * torch.exp(s["g"])[..., None, None]
        u = s["beta"].unsqueeze(-1) * (v - (k.unsqueeze(-1) * state).sum(-2))
        state = state + k.unsqueeze(-1) * u.unsqueeze(-2)
        out = (q.unsqueeze(-1) * state).sum(-2) * s["q_scale"]
        return {"out": out.to(s["v"].dtype), "state": state}
    train = s["kind"] == "delta_train"
    names = ("q", "k", "v", "g", "beta")
    leaves = [s[n].detach().float().requires_grad_(train) for n in names]
    state = state.detach().requires_grad_(train)
    none = None if s["lengths"] is None else _behind(s["lengths"], s["v"].transpose(1, 2)).squeeze(-1).transpose(1, 2)
    out, last = _plain_rule(*leaves, s["q_scale"], state, none)
    got = {"out": out.detach().to(s["v"].dtype), "state": last.detach()}
    if train:
        dlast = s["dstate_out"] if s["dstate_out"] is not None else torch.zeros_like(last)
        dout = s["dout"].float()
        if none is not None:
            dout = dout.masked_fill(none.unsqueeze(-1), 0.0)
        grads = torch.autograd.grad((out, last), leaves + [state], (dout, dlast))
        got |= {"d" + n: t.to(s[n].dtype) for n, t in zip(names, grads)}
        if s["dstate_in"] is not None:
            got["dstate"] = grads[-1]
    return got


def run(state):
    kind = state["kind"]
    if kind == "rope":
        return _own_rope(state) if own else _plain_rope(state)
    if kind.startswith("norm"):
        return _own_norm(state) if own else _plain_norm(state)
    return _own_delta(state) if own else _plain_delta(state)


# ---- work and the results in 64 bits --------------------------------------------------------------------------------


def work(case):
    kind, size = case["kind"], ITEMSIZE[case["dtype"]]
    B = case["B"]
    if kind == "rope":
        N = _tokens(case)
        values = B * N * (case["H"] + case["Hk"]) * case["d"]
        positions = 4 * len(case["channels"].split(",")) * N * (B if case["own_positions"] else 1)
        return {"bytes": 2 * values * size + positions, "flops": 3 * values}
    if kind.startswith("norm"):
        values, rows = B * case["N"] * case["C"], B * case["C"]
        if kind == "norm_fwd":   # x and f in, y and h out; three modulation rows
            return {"bytes": 4 * values * size + 12 * rows, "flops": 12 * values}
        # and dy, dh in, dx, df out; three gradients of the modulation
        return {"bytes": 8 * values * size + 24 * rows, "flops": 36 * values}
    H, Hk, N, dk, dv = (case[n] for n in ("H", "Hk", "N", "dk", "dv"))
    states = B * H * dk * dv * 4
    values = B * N * (2 * Hk * dk + 2 * H * dv) * size + 8 * B * N * H
    # a token: the state's decay, what it holds for the key, its correction, and its answer to the query
    flops = 7 * B * N * H * dk * dv
    states *= 2 if case["state"] else 1
    if kind == "delta_train":
        # dout in, five gradients out; the gradient of the state in and out
        values += B * N * (2 * Hk * dk + 2 * H * dv) * size + 8 * B * N * H
        states *= 2
        flops *= 3
    return {"bytes": values + states, "flops": flops}


def _exact_rope(s):
    positions = s["positions"] if s["positions"].dim() == 3 else s["positions"].unsqueeze(0)
    got = {}
    for name in ("q", "k"):
        y, at = s[name].double().clone(), 0
        for axis, c in enumerate(s["channels"]):
            half = c // 2
            for i in range(half):
                turn = positions[:, axis].double() * math.exp(-2.0 * i / c * math.log(BASE))
                if s["inverse"]:
                    turn = -turn
                one, two = (at + 2 * i, at + 2 * i + 1) if s["neighbours"] else (at + i, at + half + i)
                z = torch.complex(y[..., one], y[..., two]) * torch.polar(torch.ones_like(turn), turn).unsqueeze(1)
                y[..., one], y[..., two] = z.real, z.imag
            at += c
        got[name] = y
    return got


def _exact_norm(s):
    wide = lambda n: None if s[n] is None else s[n].double()
    x, f, gate, scale, shift, w_pre, w_post = (wide(n) for n in ("x", "f", "gate", "scale", "shift", "w_pre", "w_post"))
    B, N, C = x.shape
    keep = torch.ones((B, N, 1), dtype=torch.float64, device="cuda")
    if s["lengths"] is not None:
        keep = (torch.arange(N, device="cuda").view(1, N) < s["lengths"].view(B, 1)).double().unsqueeze(-1)

    def stats(t):
        mean = torch.zeros_like(t[..., :1]) if s["rms"] else t.sum(-1, keepdim=True) / C
        var = ((t - mean) ** 2).sum(-1, keepdim=True) / C
        rate = 1.0 / torch.sqrt(var + NORM_EPS)
        return (t - mean) * rate, rate

    def back(unit, rate, dunit):
        less = unit * (dunit * unit).sum(-1, keepdim=True) / C
        if not s["rms"]:
            less = less + dunit.sum(-1, keepdim=True) / C
        return (dunit - less) * rate

    a = (1.0 if w_pre is None else w_pre) * (1.0 + scale)[:, None]
    inner, inner_rate = stats(f) if s["post"] else (f, None)
    branch = inner * (w_post if s["post"] else 1.0)
    y = x + gate[:, None] * branch
    unit, rate = stats(y)
    got = {"y": y * keep, "h": (unit * a + shift[:, None]) * keep}
    if s["kind"] == "norm_train":
        dy, dh = wide("dy") * keep, wide("dh") * keep
        dyt = dy + back(unit, rate, dh * a)
        by_channel = (dh * unit).sum(1)
        got["dx"] = dyt
        dbranch = gate[:, None] * dyt
        got["df"] = back(inner, inner_rate, dbranch * w_post) if s["post"] else dbranch
        got["dgate"], got["dshift"] = (dyt * branch).sum(1), dh.sum(1)
        got["dscale"] = by_channel * (1.0 if w_pre is None else w_pre)
        if w_pre is not None:
            got["dw_pre"] = (by_channel * (1.0 + scale)).sum(0)
        if s["post"]:
            got["dw_post"] = (dbranch * inner).sum((0, 1))
    return got


def _exact_delta(s, case):
    """The recurrence, one token after the other."""
    B, H, Hk, dk, dv = (case[n] for n in ("B", "H", "Hk", "dk", "dv"))
    N, group = case["N"], H // Hk
    step = case["kind"] == "delta_step"
    train = case["kind"] == "delta_train"
    if train and N * B * H * dk * dv * 8 > 48e9:
        return None
    rows = lambda n: (s[n].unsqueeze(2) if step else s[n]).double()
    q, k = (rows(n).repeat_interleave(group, 1) for n in ("q", "k"))
    v, g, beta = rows("v"), rows("g"), rows("beta")
    keep = torch.ones((B, 1, N), dtype=torch.float64, device="cuda")
    if s.get("lengths") is not None:
        keep = (torch.arange(N, device="cuda").view(1, 1, N) < s["lengths"].view(B, 1, 1)).double()
    g, beta, scale = g * keep, beta * keep, s["q_scale"]
    # token first, and rows and columns of the state ready to be multiplied
    first = lambda t: t.permute(2, 0, 1, 3).reshape(N, B * H, t.shape[3]).contiguous()
    q, k, v = first(q * scale), first(k), first(v)
    alpha, beta = (t.permute(2, 0, 1).reshape(N, B * H, 1, 1).contiguous() for t in (torch.exp(g), beta))
    q_col, k_col = q.unsqueeze(-1), k.unsqueeze(-1)
    k_row, q_row, v_row = k.unsqueeze(-2), q.unsqueeze(-2), v.unsqueeze(-2)
    start = s["state_in"].double() if s["state_in"] is not None else torch.zeros((B, H, dk, dv), device="cuda", dtype=torch.float64)
    state = start.reshape(B * H, dk, dv)
    held = torch.empty((N, B * H, dk, dv), dtype=torch.float64, device="cuda") if train else None
    out = torch.empty((N, B * H, 1, dv), dtype=torch.float64, device="cuda")
    for t in range(N):
        state = state * alpha[t]
        state = torch.baddbmm(state, k_col[t], beta[t] * (v_row[t] - torch.bmm(k_row[t], state)))
        torch.bmm(q_row[t], state, out=out[t])
        if train:
            held[t] = state
    back = lambda t, h=H: t.reshape(N, B, h, -1).permute(1, 2, 0, 3)
    got = {"out": back(out) * keep.unsqueeze(-1), "state": state.view(B, H, dk, dv)}
    if step:
        got["out"] = got["out"][:, :, 0]
    if not train:
        return got
    dout = first(s["dout"].double() * keep.unsqueeze(-1)).unsqueeze(-2)
    dstate = torch.zeros_like(state) if s["dstate_out"] is None else s["dstate_out"].double().reshape(B * H, dk, dv)
    grads = {n: torch.empty((N, B * H, w), dtype=torch.float64, device="cuda") for n, w in (("q", dk), ("k", dk), ("v", dv))}
    dg, dbeta = (torch.empty((N, B * H), dtype=torch.float64, device="cuda") for _ in range(2))
    for t in reversed(range(N)):
        before = (held[t - 1] if t else start.reshape(B * H, dk, dv)) * alpha[t]
        left = v_row[t] - torch.bmm(k_row[t], before)
        dstate = torch.baddbmm(dstate, q_col[t], dout[t])
        du = torch.bmm(k_row[t], dstate)
        dleft = beta[t] * du
        grads["q"][t] = (held[t] * dout[t]).sum(-1) * scale
        dbeta[t] = (du * left).sum((1, 2))
        grads["v"][t] = dleft.squeeze(1)
        dbefore = dstate - k_col[t] * dleft
        grads["k"][t] = (dstate * (beta[t] * left) - before * dleft).sum(-1)
        dg[t] = (dbefore * before).sum((1, 2))
        dstate = dbefore * alpha[t]
    shared = lambda t: (back(t) * keep.unsqueeze(-1)).reshape(B, Hk, group, N, dk).sum(2)
    got |= {"dq": shared(grads["q"]), "dk": shared(grads["k"]), "dv": back(grads["v"]) * keep.unsqueeze(-1),
            "dg": back(dg).squeeze(-1) * keep, "dbeta": back(dbeta).squeeze(-1) * keep}
    if case["state"]:
        got["dstate"] = dstate.view(B, H, dk, dv)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(s)
    if case["kind"].startswith("norm"):
        return _exact_norm(s)
    return _exact_delta(s, case)

"""Independent fp64 oracle of what stands around the mixer: rotary positions with several axes, the block boundary, and the
gated delta rule with its gradients.  Written from the formulas, token by token, in numpy; test infrastructure only."""
import math

import numpy as np


def rope(x, positions, channels, bases, scales=None, neighbours=False, inverse=False):
    """x: [B, H, N, d]; positions: [axes, N] or [B, axes, N] integers."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    pos = np.asarray(positions)
    if pos.ndim == 2:
        pos = np.broadcast_to(pos, (x.shape[0],) + pos.shape)
    at = 0
    for a, c in enumerate(channels):
        for i in range(c // 2):
            theta = pos[:, a].astype(np.float64) * (1.0 if scales is None else scales[a]) * bases[a] ** (-2.0 * i / c)
            theta = (-theta if inverse else theta)[:, None, :]
            p, r = (at + 2 * i, at + 2 * i + 1) if neighbours else (at + i, at + c // 2 + i)
            y[..., p] = x[..., p] * np.cos(theta) - x[..., r] * np.sin(theta)
            y[..., r] = x[..., r] * np.cos(theta) + x[..., p] * np.sin(theta)
        at += c
    return y


def norm(t, rms, eps):
    """t over its last axis: (unit, rate)."""
    mean = 0.0 if rms else t.mean(-1, keepdims=True)
    rate = 1.0 / np.sqrt(((t - mean) ** 2).mean(-1, keepdims=True) + eps)
    return (t - mean) * rate, rate


def boundary(x, f, gate, scale, shift, w_pre, w_post, residual_scale, eps, rms, post):
    """x, f: [B, N, C]; gate, scale, shift: [B, C] or [C] or None; returns y, h."""
    row = lambda v, none: none if v is None else (v[:, None] if v.ndim == 2 else v)
    y = residual_scale * x
    if f is not None:
        inner = norm(f, rms, eps)[0] * (1.0 if w_post is None else w_post) if post else f
        y = y + row(gate, 1.0) * inner
    h = norm(y, rms, eps)[0] * (1.0 if w_pre is None else w_pre) * (1.0 + row(scale, 0.0)) + row(shift, 0.0)
    return y, h


def delta(q, k, v, g, beta, scale, state=None, lengths=None):
    """The recurrence.  q, k: [B, Hk, N, dk]; v: [B, H, N, dv]; g, beta: [B, H, N].  Returns out (0 behind a row's length),
    the last state and every token's state before its decay, for `delta_gradients`."""
    B, H, N, dv = v.shape
    Hk, dk = q.shape[1], q.shape[3]
    out = np.zeros((B, H, N, dv))
    last = np.zeros((B, H, dk, dv)) if state is None else np.array(state, dtype=np.float64)
    held = np.zeros((B, H, N, dk, dv))
    for b in range(B):
        for h in range(H):
            s = last[b, h]
            for t in range(N if lengths is None else min(max(int(lengths[b]), 0), N)):
                held[b, h, t] = s
                key, qry = k[b, h // (H // Hk), t], q[b, h // (H // Hk), t]
                s = s * math.exp(g[b, h, t])
                u = beta[b, h, t] * (v[b, h, t] - key @ s)
                s = s + np.outer(key, u)
                out[b, h, t] = scale * (qry @ s)
            last[b, h] = s
    return out, last, held


def delta_gradients(q, k, v, g, beta, scale, held, dout, dlast=None, lengths=None):
    """Gradients by going back through the recurrence: dq, dk, dv, dg, dbeta, dstate."""
    B, H, N, dv = v.shape
    Hk, dk = q.shape[1], q.shape[3]
    dq, dk_, dv_ = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    dg, dbeta = np.zeros(g.shape), np.zeros(beta.shape)
    dstate = np.zeros((B, H, dk, dv)) if dlast is None else np.array(dlast, dtype=np.float64)
    for b in range(B):
        for h in range(H):
            hk, ds = h // (H // Hk), dstate[b, h]
            for t in reversed(range(N if lengths is None else min(max(int(lengths[b]), 0), N))):
                key, qry, do = k[b, hk, t], q[b, hk, t], scale * dout[b, h, t]
                before = held[b, h, t] * math.exp(g[b, h, t])
                rest = v[b, h, t] - key @ before
                u = beta[b, h, t] * rest
                after = before + np.outer(key, u)
                dq[b, hk, t] += after @ do
                ds = ds + np.outer(qry, do)
                du = key @ ds
                dbeta[b, h, t] = du @ rest
                drest = beta[b, h, t] * du
                dv_[b, h, t] = drest
                dk_[b, hk, t] += ds @ u - before @ drest
                ds = ds - np.outer(key, drest)
                dg[b, h, t] = (ds * before).sum()
                ds = ds * math.exp(g[b, h, t])
            dstate[b, h] = ds
    return dq, dk_, dv_, dg, dbeta, dstate

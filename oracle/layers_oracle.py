"""Independent fp64 oracle of the gated linear recurrence, the linear layers and the activations kept in 8 bits.  Written from the
formulas in numpy, the recurrence token by token; test infrastructure only."""
import math

import numpy as np


def sigmoid(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def _weight(decay, weight):
    """m and dm/dg for g = -decay."""
    if weight == "norm":
        m = np.sqrt(-np.expm1(-2.0 * decay))
        with np.errstate(divide="ignore"):
            return m, np.where(m > 0, -np.exp(-2.0 * decay) / m, 0.0)
    if weight == "leaky":
        return -np.expm1(-decay), -np.exp(-decay)
    return np.ones_like(decay), np.zeros_like(decay)


def scan(x, gate, inp, rate, state=None, weight="norm", reverse=False, lengths=None):
    """x, gate, inp (or None): [B, N, C]; rate: [C].  Returns out (0 behind a row's length), the last state, and what
    `scan_gradients` goes by, among it the scale that roundings of every out are measured by: the sum, along the recurrence, of the
    terms' magnitudes, those of the decayed state weighed by how much a relative error of the decay's exponent shows."""
    B, N, C = x.shape
    s, i = sigmoid(gate), np.ones_like(x) if inp is None else sigmoid(inp)
    decay = rate * s
    a, (m, dm) = np.exp(-decay), _weight(decay, weight)
    out, before = np.zeros((B, N, C)), np.zeros((B, N, C))
    scale, scale_before, last_scale = np.zeros((B, N, C)), np.zeros((B, N, C)), np.zeros((B, C))
    last = np.zeros((B, C)) if state is None else np.array(state, dtype=np.float64)
    for b in range(B):
        n = N if lengths is None else min(max(int(lengths[b]), 0), N)
        h, e = last[b], np.zeros(C)
        for t in (range(n - 1, -1, -1) if reverse else range(n)):
            before[b, t], scale_before[b, t] = h, e
            u = m[b, t] * i[b, t] * x[b, t]
            e = a[b, t] * e + (1.0 + decay[b, t]) * a[b, t] * np.abs(h) + np.abs(u)
            h = a[b, t] * h + u
            out[b, t], scale[b, t] = h, e
        last[b], last_scale[b] = h, e
    held = {"s": s, "i": i, "a": a, "m": m, "dm": dm, "decay": decay, "before": before, "scale": scale, "scale_before": scale_before,
            "last_scale": last_scale}
    return out, last, held


def scan_gradients(x, inp, rate, held, dout, dlast=None, reverse=False, lengths=None):
    """Gradients by going back through the recurrence, and beside each the scale of its roundings."""
    B, N, C = x.shape
    s, i, a, m, dm, decay, before = (held[n] for n in ("s", "i", "a", "m", "dm", "decay", "before"))
    g = {n: np.zeros((B, N, C)) for n in ("dx", "dgate", "dinput")}
    e = {n: np.zeros((B, N, C)) for n in ("dx", "dgate", "dinput")}
    g["drate"], e["drate"] = np.zeros(C), np.zeros(C)
    g["dstate_in"] = np.zeros((B, C)) if dlast is None else np.array(dlast, dtype=np.float64)
    e["dstate_in"] = np.zeros((B, C))
    for b in range(B):
        n = N if lengths is None else min(max(int(lengths[b]), 0), N)
        E, EE = g["dstate_in"][b], np.zeros(C)
        for t in reversed(range(n - 1, -1, -1) if reverse else range(n)):
            D = dout[b, t] + E
            ED = EE + np.abs(D)
            ix, h, w = i[b, t] * x[b, t], before[b, t], a[b, t]
            by_log = D * (w * h + dm[b, t] * ix)
            mag = w * np.abs(h) + np.abs(dm[b, t] * ix)
            by_scale = ED * mag + np.abs(D) * w * held["scale_before"][b, t] + (1.0 + decay[b, t]) * np.abs(D) * mag
            g["dx"][b, t], e["dx"][b, t] = D * m[b, t] * i[b, t], (ED + np.abs(D)) * m[b, t] * i[b, t]
            g["dinput"][b, t] = D * m[b, t] * ix * (1.0 - i[b, t])
            e["dinput"][b, t] = (ED + np.abs(D)) * m[b, t] * np.abs(ix)   # (1 - i: off by a step of 1)
            g["dgate"][b, t] = -by_log * decay[b, t] * (1.0 - s[b, t])
            e["dgate"][b, t] = by_scale * decay[b, t]
            g["drate"] -= by_log * s[b, t]
            e["drate"] += by_scale * s[b, t]
            E, EE = w * D, w * EE + (1.0 + decay[b, t]) * w * np.abs(D)
        g["dstate_in"][b], e["dstate_in"][b] = E, EE
    if inp is None:
        del g["dinput"], e["dinput"]
    return g, e


def _erf(x):
    return np.vectorize(math.erf)(x)


def act(z, kind, slope=0.01):
    """act(z) and its derivative."""
    if kind == "none":
        return z, np.ones_like(z)
    if kind == "leaky":
        return np.where(z > 0, z, slope * z), np.where(z > 0, 1.0, slope)
    if kind == "silu":
        p = sigmoid(z)
        return z * p, p * (1.0 + z * (1.0 - p))
    if kind == "gelu":
        p = 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2.0))
        return z * p, p + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    p = sigmoid(2.0 * c * (z + 0.044715 * z ** 3))
    return z * p, p + z * p * (1.0 - p) * 2.0 * c * (1.0 + 3.0 * 0.044715 * z * z)


def linear(x, w, bias):
    """z, and the sum of its terms' magnitudes."""
    z, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    return (z, mag) if bias is None else (z + bias, mag + np.abs(bias))


def keep8(x):
    """codes, exponent bytes and the values they stand for; x: [..., C], any finite values (a block with others: byte 255)."""
    C = x.shape[-1]
    blocks = (C + 31) // 32
    codes, exps, back = np.zeros(x.shape, dtype=np.int8), np.zeros(x.shape[:-1] + (blocks,), dtype=np.uint8), np.zeros(x.shape)
    for q in range(blocks):
        part = x[..., 32 * q:32 * q + 32]
        most = np.abs(part).max(-1)
        fine = np.isfinite(most)
        e = np.full(most.shape, -126)
        for p in range(-126, 128):   # the least power of two that does
            e = np.where(127.0 * 2.0 ** e < most, np.maximum(e, p), e)
        e = np.where(fine, e, 128)
        scale = 2.0 ** e.astype(np.float64)
        with np.errstate(invalid="ignore"):
            c = np.where(fine[..., None], np.rint(part / scale[..., None]), 0.0)
        codes[..., 32 * q:32 * q + 32] = c.astype(np.int8)
        exps[..., q] = (e + 127).astype(np.uint8)
        back[..., 32 * q:32 * q + 32] = np.where(fine[..., None], c * scale[..., None], np.nan)
    return codes, exps, back

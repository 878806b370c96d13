"""ctypes binding of what include/linfusion.h has around the mixer: rotary positions, the block boundary with its norms and
gate, and the gated delta rule.  As in binding.py: same names, argument marshalling only, views are handed over with their
strides and nothing is copied.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import LinFusionError, _dtype_code, _stream_ptr

FLAG_ROPE_NEIGHBOURS, FLAG_ROPE_INVERSE = 1, 2
FLAG_NORM_RMS, FLAG_NORM_POST = 1, 2

_I64x2 = ctypes.c_longlong * 2
_I64x3 = ctypes.c_longlong * 3


def declare(lib) -> None:
    if not hasattr(lib, "linfusion_rope"):   # another build named by LINFUSION_LIBRARY may be older than these entry points
        return
    vp, i32, i64, f32, u32, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_uint,
                                  ctypes.c_size_t)
    lib.linfusion_rope.argtypes = [vp] * 5 + [i32] + [vp] * 3 + [i32, i32, i32, i64, i32, i32, u32, vp] + [vp] * 6
    lib.linfusion_rope.restype = i32
    lib.linfusion_gate_norm_fwd.argtypes = [vp] * 9 + [i32, i64, i32, i32, f32, f32, u32, vp, vp, i64, vp]
    lib.linfusion_gate_norm_fwd.restype = i32
    lib.linfusion_gate_norm_bwd.argtypes = [vp] * 15 + [i32, i64, i32, i32, f32, f32, u32, vp, vp, i64, i64, vp, sz, vp]
    lib.linfusion_gate_norm_bwd.restype = i32
    lib.linfusion_gate_norm_bwd_workspace_bytes.argtypes = [i32, i64, i32]
    lib.linfusion_gate_norm_bwd_workspace_bytes.restype = sz
    sizes = [i32, i32, i32, i64, i32, i32, i32]
    lib.linfusion_delta_fwd.argtypes = [vp] * 10 + [sz] + sizes + [f32, u32] + [vp] * 6 + [sz, vp]
    lib.linfusion_delta_fwd.restype = i32
    lib.linfusion_delta_bwd.argtypes = [vp] * 9 + [sz] + [vp] * 7 + sizes + [f32, u32] + [vp] * 10 + [sz, vp]
    lib.linfusion_delta_bwd.restype = i32
    for name in ("linfusion_delta_workspace_bytes", "linfusion_delta_saved_bytes", "linfusion_delta_bwd_workspace_bytes"):
        getattr(lib, name).argtypes = sizes
        getattr(lib, name).restype = sz
    lib.linfusion_delta_step.argtypes = [vp] * 8 + [i32] * 6 + [f32, u32] + [vp] * 6
    lib.linfusion_delta_step.restype = i32


def _ptr(t):
    return None if t is None else t.data_ptr()


def _size(t):
    return 0 if t is None else t.numel() * t.element_size()


def _done(rc: int, name: str, check: bool) -> int:
    if check and rc != 0:
        raise LinFusionError(rc, name)
    return rc


class _Check:
    """Shapes, types and places of a call's tensors, judged against its first one."""

    def __init__(self, first, name: str):
        if not first.is_cuda:
            raise ValueError(f"{name}: tensors must live in device memory")
        import torch
        if first.device.index != torch.cuda.current_device():
            raise ValueError(f"{name}: the tensors' device must be the current one")
        if first.dtype not in (torch.float32, torch.float16, torch.bfloat16):
            raise ValueError(f"{name} must be fp32, fp16 or bf16")
        self.device, self.dtype, self.f32, self.i32 = first.device, first.dtype, torch.float32, torch.int32

    def rows(self, name, t, shape):
        """A view of the call's type with contiguous channels."""
        if t is None:
            return None
        if tuple(t.shape) != tuple(shape) or t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"{name} must be a {list(shape)} tensor of the call's type and device")
        if shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the channels of a token must be contiguous")
        return t

    def scalars(self, name, t, shape):
        if tuple(t.shape) != tuple(shape) or t.dtype != self.f32 or t.device != self.device:
            raise ValueError(f"{name} must be an fp32 {list(shape)} tensor on the call's device")
        return t

    def vector(self, name, t, shape):
        if t is None:
            return None
        self.scalars(name, t, shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t

    def modulation(self, name, t, B, C):
        """fp32 [B, C] rows with contiguous channels, or one [C] (or [1, C]) row for the batch; its row stride."""
        if t is None:
            return None
        shared = tuple(t.shape) in ((C,), (1, C))
        if not shared and tuple(t.shape) != (B, C) or t.dtype != self.f32 or t.device != self.device:
            raise ValueError(f"{name} must be an fp32 [{B}, {C}] or [{C}] tensor on the call's device")
        if C > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: channels must be contiguous")
        return 0 if shared else t.stride(0)

    def lengths(self, t, B):
        if t is not None and (tuple(t.shape) != (B,) or t.dtype != self.i32 or t.device != self.device
                              or not t.is_contiguous()):
            raise ValueError("lengths must be a contiguous int32 tensor with one value per batch row")

    def scratch(self, name, t):
        if t is not None and (t.device != self.device or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous memory on the call's device")


def _strides3(t):
    return None if t is None else ctypes.byref(_I64x3(*t.stride()[:3]))


def linfusion_rope(q, k, q_out, k_out, positions, channels, bases, scales=None, flags: int = 0, lengths=None, stream=None,
                   check: bool = True) -> int:
    """q_out, k_out <- q, k with rotary positions.  q, q_out: [B, H, N, d] views; k, k_out: [B, H_k, N, d] views or None.
    positions: int32 [axes, N], or [B, axes, N] with positions of its own for every batch row; channels, bases and scales:
    one value per axis.  q_out may be q and k_out may be k."""
    c = _Check(q, "q")
    if q.dim() != 4 or (k is None) != (k_out is None):
        raise ValueError("q: [B, H, N, d]; k and k_out come together")
    B, H, N, d = q.shape
    Hk = 0
    c.rows("q", q, (B, H, N, d))
    c.rows("q_out", q_out, (B, H, N, d))
    if k is not None:
        Hk = k.shape[1] if k.dim() == 4 else -1
        c.rows("k", k, (B, Hk, N, d))
        c.rows("k_out", k_out, (B, Hk, N, d))
    axes = len(channels)
    if len(bases) != axes or (scales is not None and len(scales) != axes):
        raise ValueError("channels, bases and scales have one value per axis")
    if (tuple(positions.shape) not in ((axes, N), (B, axes, N)) or positions.dtype != c.i32
            or positions.device != c.device or (N > 1 and positions.stride(-1) != 1)):
        raise ValueError("positions must be an int32 [axes, N] or [B, axes, N] tensor with contiguous tokens")
    places = _I64x2(positions.stride(0) if positions.dim() == 3 else 0, positions.stride(-2))
    c.lengths(lengths, B)
    f64 = ctypes.c_double * axes
    rc = binding.library().linfusion_rope(
        q.data_ptr(), _ptr(k), q_out.data_ptr(), _ptr(k_out), positions.data_ptr(), axes, (ctypes.c_int * axes)(*channels),
        f64(*bases), None if scales is None else f64(*scales), B, H, Hk, N, d, _dtype_code(q), flags, _ptr(lengths),
        _strides3(q), _strides3(k), _strides3(q_out), _strides3(k_out), ctypes.byref(places), _stream_ptr(stream))
    return _done(rc, "linfusion_rope", check)


def _strides2(tensors):
    """{batch, token} strides of [B, N, C] views, one after the other."""
    flat = []
    for t in tensors:
        flat += [0, 0] if t is None else t.stride()[:2]
    return (ctypes.c_longlong * len(flat))(*flat)


def _one_stride(strides, what):
    known = {s for s in strides if s is not None}
    if len(known) > 1:
        raise ValueError(f"{what} must share the stride between their rows")
    return known.pop() if known else 0


def linfusion_gate_norm_fwd(x, f, gate, scale, shift, y, h, w_pre=None, w_post=None, residual_scale: float = 1.0,
                            norm_eps: float = 1e-6, flags: int = 0, lengths=None, stream=None, check: bool = True) -> int:
    """y <- residual_scale * x + gate * f (or * norm(f) * w_post: FLAG_NORM_POST), h <- norm(y) * w_pre * (1 + scale) + shift on
    [B, N, C] views.  gate, scale, shift: fp32 [B, C] rows with one stride, or [C] for the whole batch; None is 1, 0, 0.
    y or h may be None, f too; y may be x."""
    c = _Check(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = x.shape
    for name, t in (("x", x), ("f", f), ("y", y), ("h", h)):
        c.rows(name, t, (B, N, C))
    stride = _one_stride([c.modulation(n, t, B, C) for n, t in (("gate", gate), ("scale", scale), ("shift", shift))],
                         "gate, scale and shift")
    c.vector("w_pre", w_pre, (C,))
    c.vector("w_post", w_post, (C,))
    c.lengths(lengths, B)
    rc = binding.library().linfusion_gate_norm_fwd(
        x.data_ptr(), _ptr(f), _ptr(gate), _ptr(scale), _ptr(shift), _ptr(w_pre), _ptr(w_post), _ptr(y), _ptr(h), B, N, C,
        _dtype_code(x), residual_scale, norm_eps, flags, _ptr(lengths), ctypes.byref(_strides2((x, f, y, h))), stride,
        _stream_ptr(stream))
    return _done(rc, "linfusion_gate_norm_fwd", check)


def linfusion_gate_norm_bwd_workspace_bytes(B: int, N: int, C: int) -> int:
    return int(binding.library().linfusion_gate_norm_bwd_workspace_bytes(B, N, C))


def linfusion_gate_norm_bwd(x, f, gate, scale, dy, dh, dx=None, df=None, dgate=None, dscale=None, dshift=None, w_pre=None,
                            w_post=None, dw_pre=None, dw_post=None, residual_scale: float = 1.0, norm_eps: float = 1e-6,
                            flags: int = 0, lengths=None, workspace=None, stream=None, check: bool = True) -> int:
    """The gradients of linfusion_gate_norm_fwd, given those that arrive at y and h (either may be None).  Every output may be
    None; the vectors' gradients have the vectors' shapes (a [C] modulation row's is summed over the batch) and need the
    workspace.  dx may be dy."""
    c = _Check(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = x.shape
    rows = (x, f, dy, dh, dx, df)
    for name, t in zip(("x", "f", "dy", "dh", "dx", "df"), rows):
        c.rows(name, t, (B, N, C))
    stride = _one_stride([c.modulation(n, t, B, C) for n, t in (("gate", gate), ("scale", scale))], "gate and scale")
    dstride = _one_stride([c.modulation(n, t, B, C) for n, t in (("dgate", dgate), ("dscale", dscale), ("dshift", dshift))],
                          "dgate, dscale and dshift")
    if gate is None and scale is None:
        stride = dstride   # (the gradients' rows say whether the batch shares one)
    if (stride == 0) != (dstride == 0) and any(t is not None for t in (dgate, dscale, dshift)) and B > 1:
        raise ValueError("the modulation's gradients must have its shape")
    for name, t in (("w_pre", w_pre), ("w_post", w_post), ("dw_pre", dw_pre), ("dw_post", dw_post)):
        c.vector(name, t, (C,))
    c.lengths(lengths, B)
    c.scratch("workspace", workspace)
    rc = binding.library().linfusion_gate_norm_bwd(
        x.data_ptr(), _ptr(f), _ptr(gate), _ptr(scale), _ptr(w_pre), _ptr(w_post), _ptr(dy), _ptr(dh), _ptr(dx), _ptr(df),
        _ptr(dgate), _ptr(dscale), _ptr(dshift), _ptr(dw_pre), _ptr(dw_post), B, N, C, _dtype_code(x), residual_scale,
        norm_eps, flags, _ptr(lengths), ctypes.byref(_strides2(rows)), stride, dstride, _ptr(workspace), _size(workspace),
        _stream_ptr(stream))
    return _done(rc, "linfusion_gate_norm_bwd", check)


def linfusion_delta_workspace_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_workspace_bytes(B, H, H_k, N, d_k, d_v, dtype))


def linfusion_delta_saved_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_saved_bytes(B, H, H_k, N, d_k, d_v, dtype))


def linfusion_delta_bwd_workspace_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_bwd_workspace_bytes(B, H, H_k, N, d_k, d_v, dtype))


def _delta_tensors(q, k, v, g, beta):
    c = _Check(q, "q")
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k: [B, H_k, N, d_k]; v: [B, H, N, d_v]")
    B, Hk, N, dk = q.shape
    H, dv = v.shape[1], v.shape[3]
    c.rows("q", q, (B, Hk, N, dk))
    c.rows("k", k, (B, Hk, N, dk))
    c.rows("v", v, (B, H, N, dv))
    c.scalars("g", g, (B, H, N))
    c.scalars("beta", beta, (B, H, N))
    if g.stride() != beta.stride():
        raise ValueError("g and beta must share their strides")
    return c, B, H, Hk, N, dk, dv


def linfusion_delta_fwd(q, k, v, g, beta, out, scale: float = 1.0, state_in=None, state_out=None, lengths=None, saved=None,
                        workspace=None, stream=None, check: bool = True) -> int:
    """out (and state_out) <- the gated delta rule.  q, k: [B, H_k, N, d_k] views, v, out: [B, H, N, d_v] views, g (log
    decays) and beta: fp32 [B, H, N] views with one set of strides, states: contiguous fp32 [B, H, d_k, d_v].  `saved`:
    memory of linfusion_delta_saved_bytes(...) for linfusion_delta_bwd, else `workspace` of
    linfusion_delta_workspace_bytes(...)."""
    c, B, H, Hk, N, dk, dv = _delta_tensors(q, k, v, g, beta)
    c.rows("out", out, (B, H, N, dv))
    c.vector("state_in", state_in, (B, H, dk, dv))
    c.vector("state_out", state_out, (B, H, dk, dv))
    c.lengths(lengths, B)
    c.scratch("saved", saved)
    c.scratch("workspace", workspace)
    rc = binding.library().linfusion_delta_fwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), out.data_ptr(),
        _ptr(state_out), _ptr(lengths), _ptr(saved), _size(saved), B, H, Hk, N, dk, dv, _dtype_code(q), scale, 0,
        _strides3(q), _strides3(k), _strides3(v), _strides3(out), _strides3(g), _ptr(workspace), _size(workspace),
        _stream_ptr(stream))
    return _done(rc, "linfusion_delta_fwd", check)


def linfusion_delta_bwd(q, k, v, g, beta, dout, dq, dk, dv, dg, dbeta, scale: float = 1.0, state_in=None, dstate_out=None,
                        dstate_in=None, lengths=None, saved=None, workspace=None, stream=None, check: bool = True) -> int:
    """The gradients of linfusion_delta_fwd, given those of out and (or None) state_out.  dg and dbeta: fp32 [B, H, N] views with
    one set of strides.  `saved`: what the forward call with the same arguments left there; None forms it again."""
    c, B, H, Hk, N, d_k, d_v = _delta_tensors(q, k, v, g, beta)
    c.rows("dout", dout, (B, H, N, d_v))
    c.rows("dq", dq, (B, Hk, N, d_k))
    c.rows("dk", dk, (B, Hk, N, d_k))
    c.rows("dv", dv, (B, H, N, d_v))
    c.scalars("dg", dg, (B, H, N))
    c.scalars("dbeta", dbeta, (B, H, N))
    if dg.stride() != dbeta.stride():
        raise ValueError("dg and dbeta must share their strides")
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out), ("dstate_in", dstate_in)):
        c.vector(name, t, (B, H, d_k, d_v))
    c.lengths(lengths, B)
    c.scratch("saved", saved)
    c.scratch("workspace", workspace)
    rc = binding.library().linfusion_delta_bwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), dout.data_ptr(),
        _ptr(dstate_out), _ptr(saved), _size(saved), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dg.data_ptr(),
        dbeta.data_ptr(), _ptr(dstate_in), _ptr(lengths), B, H, Hk, N, d_k, d_v, _dtype_code(q), scale, 0, _strides3(q),
        _strides3(k), _strides3(v), _strides3(g), _strides3(dout), _strides3(dq), _strides3(dk), _strides3(dv),
        _strides3(dg), _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_delta_bwd", check)


def linfusion_delta_step(q, k, v, g, beta, state_in, state_out, out, scale: float = 1.0, stream=None,
                         check: bool = True) -> int:
    """One token more: q, k [B, H_k, d_k], v, out [B, H, d_v], g, beta fp32 [B, H]; state_out (may be state_in) and out <- the
    rule applied to state_in (None: zeros)."""
    c = _Check(q, "q")
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k: [B, H_k, d_k]; v: [B, H, d_v]")
    B, Hk, dk = q.shape
    H, dv = v.shape[1:]
    c.rows("q", q, (B, Hk, dk))
    c.rows("k", k, (B, Hk, dk))
    c.rows("v", v, (B, H, dv))
    c.rows("out", out, (B, H, dv))
    c.scalars("g", g, (B, H))
    c.scalars("beta", beta, (B, H))
    if g.stride() != beta.stride():
        raise ValueError("g and beta must share their strides")
    c.vector("state_in", state_in, (B, H, dk, dv))
    c.vector("state_out", state_out, (B, H, dk, dv))
    two = lambda t: ctypes.byref(_I64x2(*t.stride()[:2]))
    rc = binding.library().linfusion_delta_step(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), _ptr(state_out),
        out.data_ptr(), B, H, Hk, dk, dv, _dtype_code(q), scale, 0, two(q), two(k), two(v), two(out), two(g),
        _stream_ptr(stream))
    return _done(rc, "linfusion_delta_step", check)

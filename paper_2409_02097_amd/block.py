"""ctypes binding of what include/linfusion.h has around the mixer: rotary positions, the block boundary with its norms and
gate, and the gated delta rule.  As in binding.py: same names, argument marshalling only, views are handed over with their
strides and nothing is copied.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding
from .binding import LinFusionError, _dtype_code, _stream_ptr

FLAG_ROPE_NEIGHBOURS, FLAG_ROPE_INVERSE = 1, 2
FLAG_NORM_RMS, FLAG_NORM_POST = 1, 2


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


# What runs on every call is written for speed: where a whole call takes the device 5 us, checking six tensors through general
# helpers and building their stride arrays anew took the host 12.
_types = None


def _head(t, name: str):
    """(device index, dtype) of a call's first tensor: in device memory of the current device, of a supported type."""
    global _types
    if _types is None:
        import torch
        _types = (torch.float32, torch.float16, torch.bfloat16, torch.int32)
    dev = t.get_device() if t.is_cuda else -1
    if dev < 0:
        raise ValueError(f"{name}: tensors must live in device memory")
    if dev != _current_device():
        raise ValueError(f"{name}: the tensors' device must be the current one")
    if t.dtype not in _types[:3]:
        raise ValueError(f"{name} must be fp32, fp16 or bf16")
    return dev, t.dtype


def _current_device() -> int:
    if binding._raw_device is None:
        import torch
        return torch.cuda.current_device()
    return binding._raw_device()


def _rows(name, t, shape, head):
    """The host array of strides of a view of the call's type with contiguous channels."""
    if t.shape != shape or t.dtype is not head[1] or t.get_device() != head[0]:
        raise ValueError(f"{name} must be a {list(shape)} tensor of the call's type and device")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the channels of a token must be contiguous")
    return _longs(strides)


def _scalars(name, t, shape, head):
    if t.shape != shape or t.dtype is not _types[0] or t.get_device() != head[0]:
        raise ValueError(f"{name} must be an fp32 {list(shape)} tensor on the call's device")


def _scalars2(name, t, name2, t2, shape, head):
    """Two fp32 views that share their strides, whose host array this is."""
    _scalars(name, t, shape, head)
    _scalars(name2, t2, shape, head)
    strides = t.stride()
    if strides != t2.stride():
        raise ValueError(f"{name} and {name2} must share their strides")
    return _longs(strides)


def _vector(name, t, shape, head):
    if t is not None:
        _scalars(name, t, shape, head)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _modulation(names, tensors, B, C, head):
    """fp32 [B, C] rows with contiguous channels, or one [C] (or, where B is not 1, [1, C]) row for the batch: their stride, 0
    where the batch shares one, None without any."""
    stride = None
    for name, t in zip(names, tensors):
        if t is None:
            continue
        shape = t.shape
        shared = shape == (C,) or (shape == (1, C) and B != 1)
        if not shared and shape != (B, C) or t.dtype is not _types[0] or t.get_device() != head[0]:
            raise ValueError(f"{name} must be an fp32 [{B}, {C}] or [{C}] tensor on the call's device")
        if t.stride(-1) != 1:
            raise ValueError(f"{name}: channels must be contiguous")
        s = 0 if shared or B == 1 else t.stride(0)
        if stride is not None and s != stride:
            raise ValueError(f"{', '.join(names)} must share the stride between their rows")
        stride = s
    return stride


def _lengths(t, B, head):
    if t is not None and (t.shape != (B,) or t.dtype is not _types[3] or t.get_device() != head[0] or not t.is_contiguous()):
        raise ValueError("lengths must be a contiguous int32 tensor with one value per batch row")


def _scratch(name, t, head):
    if t is not None and (t.get_device() != head[0] or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous memory on the call's device")


@functools.lru_cache(maxsize=1024)
def _longs(values):
    """A host array of the values; read by the library during the call only."""
    return (ctypes.c_longlong * len(values))(*values)


@functools.lru_cache(maxsize=64)
def _ints(values):
    return (ctypes.c_int * len(values))(*values)


@functools.lru_cache(maxsize=64)
def _doubles(values):
    return (ctypes.c_double * len(values))(*values)


def linfusion_rope(q, k, q_out, k_out, positions, channels, bases, scales=None, flags: int = 0, lengths=None, stream=None,
                   check: bool = True) -> int:
    """q_out, k_out <- q, k with rotary positions.  q, q_out: [B, H, N, d] views; k, k_out: [B, H_k, N, d] views or None.
    positions: int32 [axes, N], or [B, axes, N] with positions of its own for every batch row; channels, bases and scales:
    one value per axis.  q_out may be q and k_out may be k."""
    head = _head(q, "q")
    if q.dim() != 4 or (k is None) != (k_out is None):
        raise ValueError("q: [B, H, N, d]; k and k_out come together")
    B, H, N, d = shape = q.shape
    Hk = 0
    sq, sqo, sk, sko = _rows("q", q, shape, head), _rows("q_out", q_out, shape, head), None, None
    if k is not None:
        Hk = k.shape[1] if k.dim() == 4 else -1
        sk = _rows("k", k, (B, Hk, N, d), head)
        sko = _rows("k_out", k_out, k.shape, head)
    axes = len(channels)
    if len(bases) != axes or (scales is not None and len(scales) != axes):
        raise ValueError("channels, bases and scales have one value per axis")
    if (positions.shape not in ((axes, N), (B, axes, N)) or positions.dtype is not _types[3]
            or positions.get_device() != head[0] or (N > 1 and positions.stride(-1) != 1)):
        raise ValueError("positions must be an int32 [axes, N] or [B, axes, N] tensor with contiguous tokens")
    places = positions.stride()
    places = places[:2] if positions.dim() == 3 else (0, places[0])
    _lengths(lengths, B, head)
    rc = binding.library().linfusion_rope(
        q.data_ptr(), _ptr(k), q_out.data_ptr(), _ptr(k_out), positions.data_ptr(), axes, _ints(tuple(channels)),
        _doubles(tuple(bases)), None if scales is None else _doubles(tuple(scales)), B, H, Hk, N, d, _dtype_code(q), flags,
        _ptr(lengths), sq, sk, sqo, sko, _longs(places), _stream_ptr(stream))
    return _done(rc, "linfusion_rope", check)


def _plain(t, shape, head) -> bool:
    return t is None or (t.shape == shape and t.dtype is head[1] and t.is_contiguous() and t.get_device() == head[0])


def _strides2(*tensors):
    """{batch, token} strides of [B, N, C] views, one after the other."""
    flat = ()
    for t in tensors:
        flat += (0, 0) if t is None else t.stride()[:2]
    return _longs(flat)


def linfusion_gate_norm_fwd(x, f, gate, scale, shift, y, h, w_pre=None, w_post=None, residual_scale: float = 1.0,
                            norm_eps: float = 1e-6, flags: int = 0, lengths=None, stream=None, check: bool = True) -> int:
    """y <- residual_scale * x + gate * f (or * norm(f) * w_post: FLAG_NORM_POST), h <- norm(y) * w_pre * (1 + scale) + shift on
    [B, N, C] views.  gate, scale, shift: fp32 [B, C] rows with one stride, or [C] for the whole batch; None is 1, 0, 0.
    y or h may be None, f too; y may be x."""
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    strides = None
    if not (_plain(x, shape, head) and _plain(f, shape, head) and _plain(y, shape, head) and _plain(h, shape, head)):
        for name, t in (("x", x), ("f", f), ("y", y), ("h", h)):
            if t is not None:
                _rows(name, t, shape, head)
        strides = _strides2(x, f, y, h)
    stride = _modulation(("gate", "scale", "shift"), (gate, scale, shift), B, C, head) or 0
    _vector("w_pre", w_pre, (C,), head)
    _vector("w_post", w_post, (C,), head)
    _lengths(lengths, B, head)
    rc = binding.library().linfusion_gate_norm_fwd(
        x.data_ptr(), _ptr(f), _ptr(gate), _ptr(scale), _ptr(shift), _ptr(w_pre), _ptr(w_post), _ptr(y), _ptr(h), B, N, C,
        _dtype_code(x), residual_scale, norm_eps, flags, _ptr(lengths), strides, stride,
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
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    rows = (x, f, dy, dh, dx, df)
    strides = None
    if not all([_plain(t, shape, head) for t in rows]):
        for name, t in zip(("x", "f", "dy", "dh", "dx", "df"), rows):
            if t is not None:
                _rows(name, t, shape, head)
        strides = _strides2(*rows)
    stride = _modulation(("gate", "scale"), (gate, scale), B, C, head)
    dstride = _modulation(("dgate", "dscale", "dshift"), (dgate, dscale, dshift), B, C, head)
    if stride is None:
        stride = dstride   # (the gradients' rows say whether the batch shares one)
    if dstride is not None and B > 1 and (stride == 0) != (dstride == 0):
        raise ValueError("the modulation's gradients must have its shape")
    for name, t in (("w_pre", w_pre), ("w_post", w_post), ("dw_pre", dw_pre), ("dw_post", dw_post)):
        _vector(name, t, (C,), head)
    _lengths(lengths, B, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_gate_norm_bwd(
        x.data_ptr(), _ptr(f), _ptr(gate), _ptr(scale), _ptr(w_pre), _ptr(w_post), _ptr(dy), _ptr(dh), _ptr(dx), _ptr(df),
        _ptr(dgate), _ptr(dscale), _ptr(dshift), _ptr(dw_pre), _ptr(dw_post), B, N, C, _dtype_code(x), residual_scale,
        norm_eps, flags, _ptr(lengths), strides, stride or 0, dstride or 0, _ptr(workspace), _size(workspace),
        _stream_ptr(stream))
    return _done(rc, "linfusion_gate_norm_bwd", check)


def linfusion_delta_workspace_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_workspace_bytes(B, H, H_k, N, d_k, d_v, dtype))


def linfusion_delta_saved_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_saved_bytes(B, H, H_k, N, d_k, d_v, dtype))


def linfusion_delta_bwd_workspace_bytes(B: int, H: int, H_k: int, N: int, d_k: int, d_v: int, dtype: int) -> int:
    return int(binding.library().linfusion_delta_bwd_workspace_bytes(B, H, H_k, N, d_k, d_v, dtype))


def _delta_tensors(q, k, v, g, beta):
    head = _head(q, "q")
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k: [B, H_k, N, d_k]; v: [B, H, N, d_v]")
    B, Hk, N, dk = q.shape
    H, dv = v.shape[1], v.shape[3]
    key = q.shape
    strides = _rows("q", q, key, head), _rows("k", k, key, head), _rows("v", v, (B, H, N, dv), head), _scalars2("g", g, "beta", beta, (B, H, N), head)
    return head, strides, B, H, Hk, N, dk, dv


def linfusion_delta_fwd(q, k, v, g, beta, out, scale: float = 1.0, state_in=None, state_out=None, lengths=None, saved=None,
                        workspace=None, stream=None, check: bool = True) -> int:
    """out (and state_out) <- the gated delta rule.  q, k: [B, H_k, N, d_k] views, v, out: [B, H, N, d_v] views, g (log
    decays) and beta: fp32 [B, H, N] views with one set of strides, states: contiguous fp32 [B, H, d_k, d_v].  `saved`:
    memory of linfusion_delta_saved_bytes(...) for linfusion_delta_bwd, else `workspace` of
    linfusion_delta_workspace_bytes(...)."""
    head, (sq, sk, sv, sg), B, H, Hk, N, dk, dv = _delta_tensors(q, k, v, g, beta)
    so = _rows("out", out, v.shape, head)
    _vector("state_in", state_in, (B, H, dk, dv), head)
    _vector("state_out", state_out, (B, H, dk, dv), head)
    _lengths(lengths, B, head)
    _scratch("saved", saved, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_delta_fwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), out.data_ptr(),
        _ptr(state_out), _ptr(lengths), _ptr(saved), _size(saved), B, H, Hk, N, dk, dv, _dtype_code(q), scale, 0,
        sq, sk, sv, so, sg, _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_delta_fwd", check)


def linfusion_delta_bwd(q, k, v, g, beta, dout, dq, dk, dv, dg, dbeta, scale: float = 1.0, state_in=None, dstate_out=None,
                        dstate_in=None, lengths=None, saved=None, workspace=None, stream=None, check: bool = True) -> int:
    """The gradients of linfusion_delta_fwd, given those of out and (or None) state_out.  dg and dbeta: fp32 [B, H, N] views with
    one set of strides.  `saved`: what the forward call with the same arguments left there; None forms it again."""
    head, (sq, sk, sv, sg), B, H, Hk, N, d_k, d_v = _delta_tensors(q, k, v, g, beta)
    sdo = _rows("dout", dout, v.shape, head)
    sdq, sdk, sdv = _rows("dq", dq, q.shape, head), _rows("dk", dk, q.shape, head), _rows("dv", dv, v.shape, head)
    sdg = _scalars2("dg", dg, "dbeta", dbeta, (B, H, N), head)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out), ("dstate_in", dstate_in)):
        _vector(name, t, (B, H, d_k, d_v), head)
    _lengths(lengths, B, head)
    _scratch("saved", saved, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_delta_bwd(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), dout.data_ptr(),
        _ptr(dstate_out), _ptr(saved), _size(saved), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dg.data_ptr(),
        dbeta.data_ptr(), _ptr(dstate_in), _ptr(lengths), B, H, Hk, N, d_k, d_v, _dtype_code(q), scale, 0, sq, sk, sv, sg, sdo,
        sdq, sdk, sdv, sdg, _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_delta_bwd", check)


def linfusion_delta_step(q, k, v, g, beta, state_in, state_out, out, scale: float = 1.0, stream=None,
                         check: bool = True) -> int:
    """One token more: q, k [B, H_k, d_k], v, out [B, H, d_v], g, beta fp32 [B, H]; state_out (may be state_in) and out <- the
    rule applied to state_in (None: zeros)."""
    head = _head(q, "q")
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k: [B, H_k, d_k]; v: [B, H, d_v]")
    B, Hk, dk = q.shape
    H, dv = v.shape[1:]
    key, val, state = q.shape, v.shape, (B, H, dk, dv)
    sq, sk, sv, so = _rows("q", q, key, head), _rows("k", k, key, head), _rows("v", v, val, head), _rows("out", out, val, head)
    sg = _scalars2("g", g, "beta", beta, (B, H), head)
    _vector("state_in", state_in, state, head)
    _vector("state_out", state_out, state, head)
    rc = binding.library().linfusion_delta_step(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), _ptr(state_in), _ptr(state_out),
        out.data_ptr(), B, H, Hk, dk, dv, _dtype_code(q), scale, 0, sq, sk, sv, so, sg, _stream_ptr(stream))
    return _done(rc, "linfusion_delta_step", check)

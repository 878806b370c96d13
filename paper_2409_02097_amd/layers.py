"""ctypes binding of the recurrent mixer, the linear layers and the activations kept in 8 bits of include/linfusion.h.  As in
block.py: same names, argument marshalling only, views are handed over with their strides and nothing is copied.
"""
from __future__ import annotations

import ctypes

from . import binding, block
from .binding import _dtype_code, _stream_ptr
from .block import _done, _head, _lengths, _longs, _plain, _ptr, _rows, _scratch, _size, _vector

FLAG_SCAN_REVERSE, FLAG_SCAN_LEAKY, FLAG_SCAN_SUM = 1, 2, 4
ACT_NONE, ACT_LEAKY_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = range(5)
KEEP_BLOCK = 32


def declare(lib) -> None:
    if not hasattr(lib, "linfusion_scan_fwd"):   # another build named by LINFUSION_LIBRARY may be older than these entry points
        return
    vp, i32, i64, f32, u32, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_uint,
                                  ctypes.c_size_t)

    def of(name, args, result=i32):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = result

    of("linfusion_scan_fwd", [vp] * 9 + [sz, i32, i64, i32, i32, u32, vp, vp, sz, vp])
    of("linfusion_scan_bwd", [vp] * 8 + [sz] + [vp] * 6 + [i32, i64, i32, i32, u32, vp, vp, sz, vp])
    of("linfusion_scan_step", [vp] * 7 + [i32, i32, i32, u32, vp, vp])
    for name in ("workspace", "saved", "bwd_workspace"):
        of(f"linfusion_scan_{name}_bytes", [i32, i64, i32], sz)
    of("linfusion_linear_fwd", [vp] * 6 + [i32, i64, i32, i32, i32, i32, f32, u32, vp, vp, i64, vp, sz, vp])
    of("linfusion_linear_bwd", [vp] * 9 + [i32, i64, i32, i32, i32, i32, f32, u32, vp, vp, i64, i64, vp, sz, vp])
    for name in ("workspace", "bwd_workspace"):
        of(f"linfusion_linear_{name}_bytes", [i32, i64, i32, i32, i32], sz)
    of("linfusion_keep8", [vp] * 3 + [i32, i64, i32, i32, u32, vp, vp, vp])
    of("linfusion_unkeep8", [vp] * 3 + [i32, i64, i32, i32, u32, vp, vp, vp])


def _tokens(named, head):
    """{batch, token} strides of [B, N, C] views of the call's type (None: absent), one after the other; None where all of them are
    contiguous."""
    for _, t, shape in named:
        if not _plain(t, shape, head):
            break
    else:
        return None
    flat = ()
    for name, t, shape in named:
        if t is None:
            flat += (0, 0)
        else:
            _rows(name, t, shape, head)
            flat += t.stride()[:2]
    return _longs(flat)


# ---- the gated linear recurrence --------------------------------------------------------------------------------------


def linfusion_scan_workspace_bytes(B: int, N: int, C: int) -> int:
    return int(binding.library().linfusion_scan_workspace_bytes(B, N, C))


def linfusion_scan_saved_bytes(B: int, N: int, C: int) -> int:
    return int(binding.library().linfusion_scan_saved_bytes(B, N, C))


def linfusion_scan_bwd_workspace_bytes(B: int, N: int, C: int) -> int:
    return int(binding.library().linfusion_scan_bwd_workspace_bytes(B, N, C))


def linfusion_scan_fwd(x, gate, input, rate, out, state_in=None, state_out=None, saved=None, lengths=None, flags: int = 0,
                       workspace=None, stream=None, check: bool = True) -> int:
    """out (and state_out) <- h = a h + m sigmoid(input) x with a = exp(-rate sigmoid(gate)), channel by channel.  x, gate, input
    (or None), out: [B, N, C] views; rate: fp32 [C]; states: contiguous fp32 [B, C].  `saved`: memory of
    linfusion_scan_saved_bytes(...) for linfusion_scan_bwd; `workspace` of linfusion_scan_workspace_bytes(...)."""
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    strides = _tokens((("x", x, shape), ("gate", gate, shape), ("input", input, shape), ("out", out, shape)), head)
    _vector("rate", rate, (C,), head)
    _vector("state_in", state_in, (B, C), head)
    _vector("state_out", state_out, (B, C), head)
    _lengths(lengths, B, head)
    _scratch("saved", saved, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_scan_fwd(
        x.data_ptr(), _ptr(gate), _ptr(input), _ptr(rate), _ptr(state_in), _ptr(out), _ptr(state_out), _ptr(lengths), _ptr(saved),
        _size(saved), B, N, C, _dtype_code(x), flags, strides, _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_scan_fwd", check)


def linfusion_scan_bwd(x, gate, input, rate, dout, dx, dgate, dinput, drate, state_in=None, dstate_out=None, dstate_in=None,
                       saved=None, lengths=None, flags: int = 0, workspace=None, stream=None, check: bool = True) -> int:
    """The gradients of linfusion_scan_fwd, given those of out and (or None) state_out.  `saved`: what the forward call with the
    same arguments left there; None forms it again.  `workspace` of linfusion_scan_bwd_workspace_bytes(...)."""
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    strides = _tokens([(n, t, shape) for n, t in (("x", x), ("gate", gate), ("input", input), ("dout", dout), ("dx", dx),
                                                  ("dgate", dgate), ("dinput", dinput))], head)
    _vector("rate", rate, (C,), head)
    _vector("drate", drate, (C,), head)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out), ("dstate_in", dstate_in)):
        _vector(name, t, (B, C), head)
    _lengths(lengths, B, head)
    _scratch("saved", saved, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_scan_bwd(
        x.data_ptr(), _ptr(gate), _ptr(input), _ptr(rate), _ptr(state_in), _ptr(dout), _ptr(dstate_out), _ptr(saved), _size(saved),
        _ptr(dx), _ptr(dgate), _ptr(dinput), _ptr(drate), _ptr(dstate_in), _ptr(lengths), B, N, C, _dtype_code(x), flags, strides,
        _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_scan_bwd", check)


def linfusion_scan_step(x, gate, input, rate, state_in, state_out, out, flags: int = 0, stream=None, check: bool = True) -> int:
    """One token more of every batch row: x, gate, input (or None), out [B, C] views; state_out (None: not kept; may be state_in)
    and out <- the recurrence from state_in (None: zeros)."""
    head = _head(x, "x")
    if x.dim() != 2:
        raise ValueError("x: [B, C]")
    B, C = shape = x.shape
    strides = None
    if not (_plain(x, shape, head) and _plain(gate, shape, head) and _plain(input, shape, head) and _plain(out, shape, head)):
        flat = ()
        for name, t in (("x", x), ("gate", gate), ("input", input), ("out", out)):
            if t is not None:
                _rows(name, t, shape, head)
            flat += (0,) if t is None else t.stride()[:1]
        strides = _longs(flat)
    _vector("rate", rate, (C,), head)
    _vector("state_in", state_in, shape, head)
    _vector("state_out", state_out, shape, head)
    rc = binding.library().linfusion_scan_step(
        x.data_ptr(), _ptr(gate), _ptr(input), _ptr(rate), _ptr(state_in), _ptr(state_out), _ptr(out), B, C, _dtype_code(x), flags,
        strides, _stream_ptr(stream))
    return _done(rc, "linfusion_scan_step", check)


# ---- linear layers ----------------------------------------------------------------------------------------------------


def linfusion_linear_workspace_bytes(B: int, N: int, C_in: int, C_out: int, dtype: int) -> int:
    return int(binding.library().linfusion_linear_workspace_bytes(B, N, C_in, C_out, dtype))


def linfusion_linear_bwd_workspace_bytes(B: int, N: int, C_in: int, C_out: int, dtype: int) -> int:
    return int(binding.library().linfusion_linear_bwd_workspace_bytes(B, N, C_in, C_out, dtype))


def _matrix(name, t, shape, head):
    """The stride between the rows of a matrix of the call's type."""
    if t.shape != shape or t.dtype is not head[1] or t.get_device() != head[0]:
        raise ValueError(f"{name} must be a {list(shape)} tensor of the call's type and device")
    if shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: a row's elements must be contiguous")
    if shape[0] > 1 and t.stride(0) < shape[1]:   # (one row for all of them has stride 0, which the library takes for contiguous rows)
        raise ValueError(f"{name}: the rows must lie one behind the other")
    return t.stride(0) if shape[0] > 1 else shape[1]


def _bias(name, t, C, head):
    if t is not None and (t.shape != (C,) or t.dtype is not head[1] or t.get_device() != head[0] or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous [{C}] tensor of the call's type and device")


def linfusion_linear_fwd(x, w, bias, y, residual=None, z=None, activation: int = ACT_NONE, slope: float = 0.01, lengths=None,
                         workspace=None, stream=None, check: bool = True) -> int:
    """z <- x w^T + bias, y <- residual + act(z).  x: [B, N, C_in] view; w: [C_out, C_in] with contiguous rows; bias: [C_out] or None;
    residual, y, z: [B, N, C_out] views or None (y or z must be there).  y may be the residual.  `workspace` of
    linfusion_linear_workspace_bytes(...)."""
    head = _head(x, "x")
    if x.dim() != 3 or w.dim() != 2:
        raise ValueError("x: [B, N, C_in]; w: [C_out, C_in]")
    B, N, K = x.shape
    C = w.shape[0]
    shape = (B, N, C)
    strides = _tokens((("x", x, x.shape), ("residual", residual, shape), ("y", y, shape), ("z", z, shape)), head)
    ws = _matrix("w", w, (C, K), head)
    _bias("bias", bias, C, head)
    _lengths(lengths, B, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_linear_fwd(
        x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(residual), _ptr(y), _ptr(z), B, N, K, C, _dtype_code(x), activation, slope, 0,
        _ptr(lengths), strides, ws, _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_linear_fwd", check)


def _kept(name, t, exps, shape, head):
    """{batch, token} strides of 8-bit codes and of their exponents."""
    import torch
    if t.shape != shape or t.dtype is not torch.int8 or t.get_device() != head[0] or t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must be an int8 {list(shape)} tensor with contiguous channels on the call's device")
    blocks = (*shape[:-1], (shape[-1] + KEEP_BLOCK - 1) // KEEP_BLOCK)
    if exps.shape != blocks or exps.dtype is not torch.uint8 or exps.get_device() != head[0] or exps.stride(-1) != 1 and blocks[-1] > 1:
        raise ValueError(f"the exponents of {name} must be a uint8 {list(blocks)} tensor with contiguous blocks on the call's device")
    return t.stride()[:2], exps.stride()[:2]


def linfusion_linear_bwd(x, w, z, dy, dx=None, dw=None, dbias=None, x_exps=None, z_exps=None, activation: int = ACT_NONE,
                         slope: float = 0.01, lengths=None, workspace=None, stream=None, check: bool = True) -> int:
    """The gradients of linfusion_linear_fwd, given dy: dx, dw, dbias, each may be None (not all).  z: the values before the activation
    (None without one).  x and z may be int8 codes that linfusion_keep8 left, with their exponents.  `workspace` of
    linfusion_linear_bwd_workspace_bytes(...)."""
    head = _head(dy, "dy")
    if dy.dim() != 3 or w.dim() != 2:
        raise ValueError("dy: [B, N, C_out]; w: [C_out, C_in]")
    B, N, C = shape = dy.shape
    K = w.shape[1]
    wide = (B, N, K)
    sxe = sze = (0, 0)
    if x_exps is not None:
        sx, sxe = _kept("x", x, x_exps, wide, head)
    else:
        sx = (0, 0) if x is None else (_rows("x", x, wide, head), x.stride()[:2])[1]
    if z_exps is not None:
        sz, sze = _kept("z", z, z_exps, shape, head)
    else:
        sz = (0, 0) if z is None else (_rows("z", z, shape, head), z.stride()[:2])[1]
    if dx is not None:
        _rows("dx", dx, wide, head)
    _rows("dy", dy, shape, head)
    strides = _longs((*sx, *sz, *dy.stride()[:2], *((0, 0) if dx is None else dx.stride()[:2]), *sxe, *sze))
    ws = _matrix("w", w, (C, K), head)
    dws = 0 if dw is None else _matrix("dw", dw, (C, K), head)
    _bias("dbias", dbias, C, head)
    _lengths(lengths, B, head)
    _scratch("workspace", workspace, head)
    rc = binding.library().linfusion_linear_bwd(
        _ptr(x), _ptr(x_exps), w.data_ptr(), _ptr(z), _ptr(z_exps), dy.data_ptr(), _ptr(dx), _ptr(dw), _ptr(dbias), B, N, K, C,
        _dtype_code(dy), activation, slope, 0, _ptr(lengths), strides, ws, dws, _ptr(workspace), _size(workspace), _stream_ptr(stream))
    return _done(rc, "linfusion_linear_bwd", check)


# ---- activations in 8 bits --------------------------------------------------------------------------------------------


def linfusion_keep8(x, codes, exps, lengths=None, stream=None, check: bool = True) -> int:
    """codes (int8 [B, N, C]), exps (uint8 [B, N, ceil(C / 32)]) <- x, a [B, N, C] view: an 8-bit integer a value, a power of two for 32
    neighbouring channels."""
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    _rows("x", x, shape, head)
    sc, se = _kept("codes", codes, exps, shape, head)
    _lengths(lengths, B, head)
    rc = binding.library().linfusion_keep8(x.data_ptr(), codes.data_ptr(), exps.data_ptr(), B, N, C, _dtype_code(x), 0, _ptr(lengths),
                                           _longs((*x.stride()[:2], *sc, *se)), _stream_ptr(stream))
    return _done(rc, "linfusion_keep8", check)


def linfusion_unkeep8(codes, exps, x, lengths=None, stream=None, check: bool = True) -> int:
    """x, a [B, N, C] view <- the values that linfusion_keep8's codes and exponents stand for."""
    head = _head(x, "x")
    if x.dim() != 3:
        raise ValueError("x: [B, N, C]")
    B, N, C = shape = x.shape
    _rows("x", x, shape, head)
    sc, se = _kept("codes", codes, exps, shape, head)
    _lengths(lengths, B, head)
    rc = binding.library().linfusion_unkeep8(codes.data_ptr(), exps.data_ptr(), x.data_ptr(), B, N, C, _dtype_code(x), 0, _ptr(lengths),
                                             _longs((*sc, *se, *x.stride()[:2])), _stream_ptr(stream))
    return _done(rc, "linfusion_unkeep8", check)

"""Operators for training and serving residual encoders (include/neuroute_ops.h):
the linear layer with its epilogue, the layer norm, the norms around a block fused
with its gate and residual scale, their gradients, activation checkpoints held in
8 bits, and the AdamW step over all parameters, its averages in 32 or 8 bits.

Argument checks and marshalling only; every step runs in the library's
kernels and there is no fallback. Matrices are CUDA tensors of two dimensions
with any row pitch (stride(1) == 1); a wrong tensor raises before any call.
Work goes to the current stream of the tensors' device, or to `stream`, on
which the outputs are then allocated (the caller orders the streams, as for any
tensor used on another than its own). Nothing synchronises, and a CUDA graph may
capture the calls. The outputs carry no autograd history; residual.py wraps the
calls in autograd functions.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional

import torch

from . import neuroute as _nr

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_DT = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_GROUP = 32  # columns that share a checkpoint's scale
_MOST = torch.finfo(torch.float32).max
_LINEAR = struct.Struct("27q")
_NORM = struct.Struct("4qd17q")
NORMS = {"none": 0, "rms": 1, "layer": 2}
GATES = {"sigmoid": 4, "silu": 3}
_BLOCK = struct.Struct("9q2d31q")
_TENSOR = struct.Struct("4qd")
_ADAMW = struct.Struct("12qdq4d2q")


class Checkpoint8:
    """A matrix held in 8 bits (nr_checkpoint8_write): codes int8 [m x 32 ceil(n / 32)],
    scales uint8 [m x ceil(n / 32)], and the shape and dtype it was made from."""

    __slots__ = ("codes", "scales", "shape", "dtype")

    def __init__(self, codes, scales, shape, dtype):
        m, n = (int(v) for v in shape)
        g = -(-n // _GROUP)
        if dtype not in _DT:
            raise ValueError(f"dtype: {dtype}, expected {' or '.join(map(str, _DT))}")
        for t, name, dt, cols in ((codes, "codes", torch.int8, g * _GROUP), (scales, "scales", torch.uint8, g)):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
            if t.dtype != dt or t.shape != (m, cols) or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"{name}: expected a contiguous CUDA tensor {dt} of shape {(m, cols)}")
        if codes.device != scales.device or codes.data_ptr() % 16:
            raise ValueError("codes and scales: on one device, codes 16-byte aligned")
        self.codes, self.scales, self.shape, self.dtype = codes, scales, (m, n), dtype

    @property
    def device(self):
        return self.codes.device

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()

    def record_stream(self, stream):
        self.codes.record_stream(stream)
        self.scales.record_stream(stream)


_HALF = (torch.float16, torch.bfloat16)
_FLOATS = tuple(_DT)
_stream = torch._C._cuda_getCurrentRawStream  # the current stream of a device index, as an integer
_address, _contiguous = torch.Tensor.data_ptr, torch.Tensor.is_contiguous


def _fail(t, name, dtypes, rows, cols, index):
    """Says what is wrong with a matrix, in the order type, dtype, shape, device, strides."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({'any' if rows is None else rows}, "
                         f"{'any' if cols is None else cols})")
    if not t.is_cuda or (index is not None and t.get_device() != index):
        raise ValueError(f"{name}: expected a tensor on {'a CUDA device' if index is None else f'cuda:{index}'}, "
                         f"got {t.device}")
    if t.shape[1] < 1 or t.shape[1] >= 1 << 24:
        raise ValueError(f"{name}: widths from 1 to 2^24 - 1 are supported, got {t.shape[1]}")
    raise ValueError(f"{name}: rows must be contiguous (stride(1) == 1)")


def _first(t, name, dtypes):
    """Checks the row-major matrix that sets a call's sizes; (rows, columns, pitch, device index)."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.is_cuda and t.dim() == 2:
        m, n = t.shape
        ld, inner = t.stride()
        if 0 < n < 16777216 and (inner == 1 or n == 1 or m == 0):
            return m, n, ld, t.get_device()
    _fail(t, name, dtypes, None, None, None)


def _matrix(t, name, dtypes, rows, cols, index):
    """Checks another matrix of the call; its row pitch in elements."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.get_device() == index and t.shape == (rows, cols):
        ld, inner = t.stride()
        if inner == 1 or cols == 1 or rows == 0:
            return ld
    _fail(t, name, dtypes, rows, cols, index)


def _vector(t, name, dtypes, n, index):
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.shape != (n,):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({n},)")
    if t.get_device() != index:
        raise ValueError(f"{name}: expected a tensor on cuda:{index}, got {t.device}")
    if n > 1 and t.stride() != (1,):
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _held(c, name, rows, cols, index, dtype):
    if c.shape != (rows, cols):
        raise ValueError(f"{name}: shape {c.shape}, expected ({rows}, {cols})")
    if c.codes.get_device() != index:
        raise ValueError(f"{name}: expected a checkpoint on cuda:{index}, got {c.device}")
    if c.dtype is not dtype:
        raise ValueError(f"{name}: made from {c.dtype}, expected {dtype}")


def _act(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"act: {name!r}, expected one of {', '.join(ACTIVATIONS)}") from None


def _elsewhere(fn, stream, args, kw):
    """fn on another stream: outputs and scratch belong to it, inputs stay alive for it."""
    with torch.cuda.stream(stream):
        out = fn(*args, **kw)
    for t in list(args) + list(kw.values()):
        if isinstance(t, Checkpoint8) or (isinstance(t, torch.Tensor) and t.is_cuda):
            t.record_stream(stream)
    return out


def _scratch(call, nbytes, device):
    """Scratch of a call and its address."""
    if nbytes <= 0:
        if nbytes < 0:
            raise _nr.NRError(call, nbytes)
        return None, 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr()


def _new_checkpoint(m, n, dtype, device):
    g = -(-n // _GROUP)
    c = Checkpoint8.__new__(Checkpoint8)
    c.codes = torch.empty((m, g * _GROUP), dtype=torch.int8, device=device)
    c.scales = torch.empty((m, g), dtype=torch.uint8, device=device)
    c.shape, c.dtype = (m, n), dtype
    return c


def checkpoint8(x, stream=None) -> Checkpoint8:
    """x [m x n] (fp32, fp16 or bf16) held in 8 bits (nr_checkpoint8_write)."""
    if stream is not None:
        return _elsewhere(checkpoint8, stream, (x,), {})
    m, n, ld, index = _first(x, "x", _FLOATS)
    c = _new_checkpoint(m, n, x.dtype, x.device)
    st = _nr.lib().nr_checkpoint8_write(x.data_ptr(), _DT[x.dtype], m, n, ld, c.codes.data_ptr(),
                                        c.scales.data_ptr(), index, _stream(index))
    if st:
        raise _nr.NRError("nr_checkpoint8_write", st)
    return c


def checkpoint8_read(c: Checkpoint8, act="none", stream=None):
    """act(the values c stands for) in the dtype it was made from (nr_checkpoint8_read)."""
    if stream is not None:
        return _elsewhere(checkpoint8_read, stream, (c,), {"act": act})
    if not isinstance(c, Checkpoint8):
        raise TypeError(f"c: expected a Checkpoint8, got {type(c).__name__}")
    a = _act(act)
    m, n = c.shape
    y = torch.empty((m, n), dtype=c.dtype, device=c.device)
    index = c.codes.get_device()
    st = _nr.lib().nr_checkpoint8_read(c.codes.data_ptr(), c.scales.data_ptr(), m, n, a, y.data_ptr(),
                                       _DT[c.dtype], n, index, _stream(index))
    if st:
        raise _nr.NRError("nr_checkpoint8_read", st)
    return y


def linear(x, w, bias=None, act="none", residual=None, save=None, out_dtype=None, stream=None):
    """y = act(x w^T + bias) + residual (nr_linear_forward).

    x [m x k], w [n x k] and residual [m x n] in fp16 or bf16; bias [n] in
    that dtype or fp32; y [m x n] in x's dtype or, with
    out_dtype=torch.float32, in fp32. save: "z" returns (y, z) with z =
    x w^T + bias, "z8" returns (y, z held in 8 bits); both are what
    linear_backward takes as z."""
    if stream is not None:
        return _elsewhere(linear, stream, (x, w, bias),
                          {"act": act, "residual": residual, "save": save, "out_dtype": out_dtype})
    m, k, x_ld, index = _first(x, "x", _HALF)
    dt, dev = x.dtype, x.device
    n = w.shape[0] if isinstance(w, torch.Tensor) and w.dim() == 2 else None
    w_ld = _matrix(w, "w", (dt,), n, k, index)
    if not 0 < n < 16777216:
        raise ValueError(f"w: widths from 1 to 2^24 - 1 are supported, got {n}")
    b = _vector(bias, "bias", (dt, torch.float32), n, index)
    a = _act(act)
    r = r_ld = z_ptr = z_scale = 0
    if residual is not None:
        r_ld, r = _matrix(residual, "residual", (dt,), m, n, index), residual.data_ptr()
    ydt = dt if out_dtype is None else out_dtype
    if ydt is not dt and ydt is not torch.float32:
        raise ValueError(f"out_dtype: {out_dtype}, expected {dt} or torch.float32")
    y = torch.empty((m, n), dtype=ydt, device=dev)
    if save == "z":
        z = torch.empty((m, n), dtype=dt, device=dev)
        z_ptr = z.data_ptr()
    elif save == "z8":
        z = _new_checkpoint(m, n, dt, dev)
        z_ptr, z_scale = z.codes.data_ptr(), z.scales.data_ptr()
    elif save is not None:
        raise ValueError(f"save: {save!r}, expected None, 'z' or 'z8'")
    if m:
        code = _DT[dt]
        packed = _LINEAR.pack(m, k, n, code, _DT[ydt], _DT[bias.dtype] if b else code, a, x.data_ptr(), x_ld, 0, 0,
                              w.data_ptr(), w_ld, b, r, r_ld, y.data_ptr(), n, z_ptr, n, z_scale, 0, 0, 0, 0, 0, 0)
        lib = _nr.lib()
        nbytes = lib.nr_linear_forward_workspace(packed, index)
        ws, ws_ptr = _scratch("nr_linear_forward", nbytes, dev)
        st = lib.nr_linear_forward(packed, index, ws_ptr, nbytes, _stream(index))
        if st:
            raise _nr.NRError("nr_linear_forward", st)
    return y if save is None else (y, z)


def linear_backward(dy, x, w, z=None, act="none", x_act="none", bias_dtype=None, need=(True, True, True),
                    stream=None):
    """(dx, dw, dbias) of linear (nr_linear_backward); the residual's gradient is dy.

    dy [m x n] in w's dtype or fp32; x [m x k] and z [m x n] (not needed when
    act is "none") as tensors in w's dtype or as Checkpoint8; x_act: with a
    Checkpoint8, the layer's input is x_act(the values it stands for).
    bias_dtype: of dbias, w's dtype or fp32 (the default). need: which of the
    three to compute, None for the others."""
    if stream is not None:
        return _elsewhere(linear_backward, stream, (dy, x, w),
                          {"z": z, "act": act, "x_act": x_act, "bias_dtype": bias_dtype, "need": need})
    n, k, w_ld, index = _first(w, "w", _HALF)
    if not 0 < n < 16777216:
        raise ValueError(f"w: widths from 1 to 2^24 - 1 are supported, got {n}")
    dt, dev = w.dtype, w.device
    m = dy.shape[0] if isinstance(dy, torch.Tensor) and dy.dim() == 2 else None
    dy_ld = _matrix(dy, "dy", (dt, torch.float32), m, n, index)
    x_scale = x_ld = z_ptr = z_ld = z_scale = 0
    if isinstance(x, Checkpoint8):
        _held(x, "x", m, k, index, dt)
        x_ptr, x_scale = x.codes.data_ptr(), x.scales.data_ptr()
    else:
        x_ld, x_ptr = _matrix(x, "x", (dt,), m, k, index), x.data_ptr()
        if x_act != "none":
            raise ValueError("x_act: only for an x held in 8 bits")
    a = _act(act)
    if a:
        if z is None:
            raise ValueError("z: needed with an activation (linear's save='z' or 'z8')")
        if isinstance(z, Checkpoint8):
            _held(z, "z", m, n, index, dt)
            z_ptr, z_scale = z.codes.data_ptr(), z.scales.data_ptr()
        else:
            z_ld, z_ptr = _matrix(z, "z", (dt,), m, n, index), z.data_ptr()
    bdt = torch.float32 if bias_dtype is None else bias_dtype
    if bdt is not dt and bdt is not torch.float32:
        raise ValueError(f"bias_dtype: {bias_dtype}, expected {dt} or torch.float32")
    dx = dw = db = None
    dx_ptr = dw_ptr = db_ptr = 0
    if need[0]:
        dx = torch.empty((m, k), dtype=dt, device=dev)
        dx_ptr = dx.data_ptr()
    if need[1]:
        dw = torch.empty((n, k), dtype=dt, device=dev)
        dw_ptr = dw.data_ptr()
    if need[2]:
        db = torch.empty(n, dtype=bdt, device=dev)
        db_ptr = db.data_ptr()
    packed = _LINEAR.pack(m, k, n, _DT[dt], _DT[dy.dtype], _DT[bdt], a, x_ptr, x_ld, x_scale, _act(x_act),
                          w.data_ptr(), w_ld, 0, 0, 0, 0, 0, z_ptr, z_ld, z_scale, dy.data_ptr(), dy_ld, dx_ptr, k,
                          dw_ptr, db_ptr)
    lib = _nr.lib()
    nbytes = lib.nr_linear_backward_workspace(packed, index)
    ws, ws_ptr = _scratch("nr_linear_backward", nbytes, dev)
    st = lib.nr_linear_backward(packed, index, ws_ptr, nbytes, _stream(index))
    if st:
        raise _nr.NRError("nr_linear_backward", st)
    return dx, dw, db


def layer_norm(x, weight=None, bias=None, eps=1e-5, save=False, stream=None):
    """y = (x - mean) rstd weight + bias over the rows of x [m x n]
    (nr_layer_norm_forward), in x's dtype (fp32, fp16 or bf16; a Checkpoint8:
    the one it was made from); weight and bias [n] in that dtype or fp32, both
    the same. save: returns (y, mean, rstd), mean and rstd [m] fp32."""
    if stream is not None:
        return _elsewhere(layer_norm, stream, (x, weight, bias), {"eps": eps, "save": save})
    x_scale = x_ld = 0
    if isinstance(x, Checkpoint8):
        m, n = x.shape
        index = x.codes.get_device()
        x_ptr, x_scale = x.codes.data_ptr(), x.scales.data_ptr()
    else:
        m, n, x_ld, index = _first(x, "x", _FLOATS)
        x_ptr = x.data_ptr()
    dt, dev = x.dtype, x.device
    wdt = weight.dtype if isinstance(weight, torch.Tensor) else bias.dtype if isinstance(bias, torch.Tensor) else dt
    w = _vector(weight, "weight", (dt, torch.float32), n, index)
    b = _vector(bias, "bias", (wdt,) if w else (dt, torch.float32), n, index)
    if not eps > 0.0:
        raise ValueError(f"eps: {eps}, expected a positive number")
    y = torch.empty((m, n), dtype=dt, device=dev)
    mean_ptr = rstd_ptr = 0
    if save:
        mean = torch.empty(m, dtype=torch.float32, device=dev)
        rstd = torch.empty(m, dtype=torch.float32, device=dev)
        mean_ptr, rstd_ptr = mean.data_ptr(), rstd.data_ptr()
    packed = _NORM.pack(m, n, _DT[dt], _DT[wdt], eps, x_ptr, x_ld, x_scale, w, b, y.data_ptr(), n, mean_ptr, rstd_ptr,
                        0, 0, 0, 0, 0, 0, 0, 0)
    if m:
        st = _nr.lib().nr_layer_norm_forward(packed, index, _stream(index))
        if st:
            raise _nr.NRError("nr_layer_norm_forward", st)
    return (y, mean, rstd) if save else y


def layer_norm_backward(dy, x, weight, mean, rstd, residual_grad=None, param_grads=True, stream=None):
    """(dx, dweight, dbias) of layer_norm (nr_layer_norm_backward); x [m x n] a
    tensor in dy's dtype or a Checkpoint8 made from that dtype, mean and rstd as
    layer_norm saved them. residual_grad [m x n] is added to dx (the gradient
    that a skip around the norm brings). weight None: ones. dweight and dbias
    have weight's dtype (fp32 without one); param_grads False: None both."""
    if stream is not None:
        return _elsewhere(layer_norm_backward, stream, (dy, x, weight, mean, rstd),
                          {"residual_grad": residual_grad, "param_grads": param_grads})
    m, n, dy_ld, index = _first(dy, "dy", _FLOATS)
    dt, dev = dy.dtype, dy.device
    x_scale = x_ld = r = r_ld = 0
    if isinstance(x, Checkpoint8):
        _held(x, "x", m, n, index, dt)
        x_ptr, x_scale = x.codes.data_ptr(), x.scales.data_ptr()
    else:
        x_ld, x_ptr = _matrix(x, "x", (dt,), m, n, index), x.data_ptr()
    w = _vector(weight, "weight", (dt, torch.float32), n, index)
    if mean is None or rstd is None:
        raise ValueError("mean, rstd: needed (layer_norm's save=True)")
    mean_ptr = _vector(mean, "mean", (torch.float32,), m, index)
    rstd_ptr = _vector(rstd, "rstd", (torch.float32,), m, index)
    if residual_grad is not None:
        r_ld, r = _matrix(residual_grad, "residual_grad", (dt,), m, n, index), residual_grad.data_ptr()
    wdt = torch.float32 if weight is None else weight.dtype
    dx = torch.empty((m, n), dtype=dt, device=dev)
    dw = db = None
    dw_ptr = db_ptr = 0
    if param_grads:
        dw = torch.empty(n, dtype=wdt, device=dev)
        db = torch.empty(n, dtype=wdt, device=dev)
        dw_ptr, db_ptr = dw.data_ptr(), db.data_ptr()
    packed = _NORM.pack(m, n, _DT[dt], _DT[wdt], 0.0, x_ptr, x_ld, x_scale, w, 0, 0, 0, mean_ptr, rstd_ptr,
                        dy.data_ptr(), dy_ld, r, r_ld, dx.data_ptr(), n, dw_ptr, db_ptr)
    lib = _nr.lib()
    nbytes = lib.nr_layer_norm_backward_workspace(packed, index)
    ws, ws_ptr = _scratch("nr_layer_norm_backward", nbytes, dev)
    st = lib.nr_layer_norm_backward(packed, index, ws_ptr, nbytes, _stream(index))
    if st:
        raise _nr.NRError("nr_layer_norm_backward", st)
    return dx, dw, db


def _named(name, what, among):
    try:
        return among[name]
    except (KeyError, TypeError):
        raise ValueError(f"{what}: {name!r}, expected one of {', '.join(among)}") from None


def _block(n, index, dt, u, gate, gate_act, scale, post, post_weight, post_bias, pre, weight, bias, m):
    """Checks what block_norm and its backward pass share: kinds, pitches, addresses and the vectors' dtype."""
    post, pre, act = _named(post, "post", NORMS), _named(pre, "pre", NORMS), _named(gate_act, "gate_act", GATES)
    u_ld = u_ptr = gate_ld = gate_ptr = gate_cols = 0
    if u is not None:
        u_ld, u_ptr = _matrix(u, "u", (dt,), m, n, index), u.data_ptr()
    elif gate is not None or scale is not None or post or not pre:
        raise ValueError("u: needed with a gate, a scale or a norm after the block, and without one before the next")
    if gate is not None:
        gate_cols = 1 if isinstance(gate, torch.Tensor) and gate.dim() == 2 and gate.shape[1] == 1 else n
        gate_ld, gate_ptr = _matrix(gate, "gate", (dt,), m, gate_cols, index), gate.data_ptr()
    if not post and (post_weight is not None or post_bias is not None):
        raise ValueError("post_weight, post_bias: only with a norm after the block (post)")
    if not pre and (weight is not None or bias is not None):
        raise ValueError("weight, bias: only with a norm before the next block (pre)")
    pointers, vdt = [], None
    for v in (scale, post_weight, post_bias, weight, bias):
        if v is None:
            pointers.append(0)
            continue
        if vdt is None and isinstance(v, torch.Tensor) and (v.dtype is dt or v.dtype is torch.float32):
            vdt = v.dtype
        if not (isinstance(v, torch.Tensor) and v.dtype is vdt and v.dim() == 1 and v.numel() == n and
                v.get_device() == index and v.is_contiguous()):  # says what is wrong
            for t, k in ((scale, "scale"), (post_weight, "post_weight"), (post_bias, "post_bias"), (weight, "weight"),
                         (bias, "bias")):
                _vector(t, k, (dt, torch.float32) if vdt is None else (vdt,), n, index)
        pointers.append(v.data_ptr())
    return (post, pre, act, gate_cols, u_ptr, u_ld, gate_ptr, gate_ld, torch.float32 if vdt is None else vdt, pointers)


def _new(like, ld, m, n, dtype, device):
    """An uninitialised contiguous [m x n]; the shorter way where `like` is one."""
    return torch.empty_like(like) if ld == n and like.dtype is dtype else torch.empty(m, n, dtype=dtype, device=device)


def block_norm(r, u=None, gate=None, gate_act="sigmoid", scale=None, alpha=1.0, post="none", post_weight=None,
               post_bias=None, pre="layer", weight=None, bias=None, eps=1e-5, save=False, out_dtype=None, stream=None):
    """(y, h) between two blocks of a residual encoder (nr_block_norm_forward):
    y = alpha r + scale gate_act(gate) (post(u) post_weight + post_bias), the residual stream after a block
    with output u, and h = pre(y) weight + bias, the next block's input.

    post and pre: "none", "rms" or "layer"; without pre h is None. u [m x n] and gate [m x n] or [m x 1] (its
    argument) in fp32, fp16 or bf16; r [m x n] in that dtype or fp32. The vectors [n] in u's dtype or fp32, all the
    same; each may be None. Without u, y is r itself and h, in out_dtype (r's by default), pre(r) weight +
    bias. save: (y, h, stats), stats what block_norm_backward takes (None where there is no norm). Backward has a 16-bit
    y only as rounded; streams whose mean is large beside their deviation are for fp32."""
    if stream is not None:
        return _elsewhere(block_norm, stream, (r, u),
                          {"gate": gate, "gate_act": gate_act, "scale": scale, "alpha": alpha, "post": post,
                           "post_weight": post_weight, "post_bias": post_bias, "pre": pre, "weight": weight,
                           "bias": bias, "eps": eps, "save": save, "out_dtype": out_dtype})
    m, n, r_ld, index = _first(r, "r", _FLOATS)
    dt = u.dtype if isinstance(u, torch.Tensor) else r.dtype if out_dtype is None else out_dtype
    if dt not in _DT:
        raise ValueError(f"{'out_dtype' if u is None else 'u'}: dtype {dt}, expected {' or '.join(map(str, _DT))}")
    if out_dtype is not None and out_dtype is not dt:
        raise ValueError(f"out_dtype: {out_dtype}, expected u's {dt}")
    if r.dtype is not dt and r.dtype is not torch.float32:
        raise ValueError(f"r: dtype {r.dtype}, expected {dt} or torch.float32")
    kpost, kpre, act, gate_cols, u_ptr, u_ld, gate_ptr, gate_ld, vdt, vectors = _block(
        n, index, dt, u, gate, gate_act, scale, post, post_weight, post_bias, pre, weight, bias, m)
    if not eps > 0.0:
        raise ValueError(f"eps: {eps}, expected a positive number")
    if not abs(alpha) <= _MOST:
        raise ValueError(f"alpha: {alpha}, expected a finite number of fp32's range")
    if u is None and alpha != 1.0:
        raise ValueError("alpha: only with u")
    dev = r.device
    y = _new(r, r_ld, m, n, r.dtype, dev) if u is not None else r
    h = (_new(r, r_ld, m, n, dt, dev) if u is None else _new(u, u_ld, m, n, dt, dev)) if kpre else None
    stats = torch.empty(kpost + kpre, m, dtype=torch.float32, device=dev) if save and kpost + kpre else None
    if m:
        packed = _BLOCK.pack(m, n, _DT[dt], _DT[r.dtype], _DT[vdt], kpost, kpre, act, gate_cols, alpha, eps, r.data_ptr(), r_ld,
                             u_ptr, u_ld, gate_ptr, gate_ld, *vectors, y.data_ptr() if u_ptr else 0, n,
                             h.data_ptr() if kpre else 0, n, 0 if stats is None else stats.data_ptr(),
                             0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        st = _nr.lib().nr_block_norm_forward(packed, index, _stream(index))
        if st:
            raise _nr.NRError("nr_block_norm_forward", st)
    return (y, h, stats) if save else (y, h)


class BlockGrads(NamedTuple):
    """Gradients of block_norm's inputs; None for what was not there."""

    r: torch.Tensor
    u: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]
    post_weight: Optional[torch.Tensor]
    post_bias: Optional[torch.Tensor]
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]


def block_norm_backward(dh, dy, y, u=None, stats=None, gate=None, gate_act="sigmoid", scale=None, alpha=1.0,
                        post="none", post_weight=None, post_bias=None, pre="layer", weight=None, bias=None,
                        param_grads=True, stream=None) -> BlockGrads:
    """Gradients of block_norm's inputs (nr_block_norm_backward), from those of its outputs: dh [m x n] in u's
    dtype (None without pre) and dy [m x n] in y's (None: zeros, with pre only). y (without pre it may be None) and
    stats as block_norm returned them, the others as it took them. The vectors' gradients have the vectors'
    dtype; param_grads False: None for all of them."""
    if stream is not None:
        return _elsewhere(block_norm_backward, stream, (dh, dy, y, u, stats),
                          {"gate": gate, "gate_act": gate_act, "scale": scale, "alpha": alpha, "post": post,
                           "post_weight": post_weight, "post_bias": post_bias, "pre": pre, "weight": weight,
                           "bias": bias, "param_grads": param_grads})
    if pre != "none":
        m, n, dh_ld, index = _first(dh, "dh", _FLOATS)
        dt, dh_ptr = dh.dtype, dh.data_ptr()
        y_ld = _matrix(y, "y", (dt, torch.float32), m, n, index)
        rdt, y_ptr, dy_ptr, dy_ld = y.dtype, y.data_ptr(), 0, 0
        if dy is not None:
            dy_ld, dy_ptr = _matrix(dy, "dy", (rdt,), m, n, index), dy.data_ptr()
    else:
        if dh is not None:
            raise ValueError("dh: only with a norm before the next block (pre)")
        m, n, dy_ld, index = _first(dy, "dy", _FLOATS)
        rdt, dy_ptr, y_ptr, y_ld, dh_ptr, dh_ld = dy.dtype, dy.data_ptr(), 0, 0, 0, 0
        dt = u.dtype if isinstance(u, torch.Tensor) and u.dtype in _DT else rdt
        if rdt is not dt and rdt is not torch.float32:
            raise ValueError(f"dy: dtype {rdt}, expected {dt} or torch.float32")
    kpost, kpre, act, gate_cols, u_ptr, u_ld, gate_ptr, gate_ld, vdt, vectors = _block(
        n, index, dt, u, gate, gate_act, scale, post, post_weight, post_bias, pre, weight, bias, m)
    if not abs(alpha) <= _MOST:
        raise ValueError(f"alpha: {alpha}, expected a finite number of fp32's range")
    if u is None and alpha != 1.0:
        raise ValueError("alpha: only with u")
    stats_ptr = 0
    if kpost + kpre:
        if stats is None:
            raise ValueError("stats: needed (block_norm's save=True)")
        ld = _matrix(stats, "stats", (torch.float32,), kpost + kpre, m, index)
        if m and ld != m and kpost + kpre > 1:
            raise ValueError("stats: must be contiguous")
        stats_ptr = stats.data_ptr()
    dev = (dh if kpre else dy).device
    first, first_ld = (dh, dh_ld) if kpre else (dy, dy_ld)
    dr = _new(first, first_ld, m, n, rdt, dev)
    du = _new(u, u_ld, m, n, dt, dev) if u is not None else None
    dgate = torch.empty(m, gate_cols, dtype=dt, device=dev) if gate is not None else None
    params = [torch.empty(n, dtype=vdt, device=dev) if param_grads and v is not None else None
              for v in (scale, post_weight, post_bias, weight, bias)]
    packed = _BLOCK.pack(m, n, _DT[dt], _DT[rdt], _DT[vdt], kpost, kpre, act, gate_cols, alpha, 0.0, 0, 0,
                         u_ptr, u_ld, gate_ptr, gate_ld, *vectors, y_ptr, y_ld, 0, 0, stats_ptr, dh_ptr, dh_ld, dy_ptr, dy_ld,
                         dr.data_ptr(), n, 0 if du is None else du.data_ptr(), n,
                         0 if dgate is None else dgate.data_ptr(), gate_cols, *[0 if p is None else p.data_ptr() for p in params])
    lib = _nr.lib()
    nbytes = lib.nr_block_norm_backward_workspace(packed, index)
    ws, ws_ptr = _scratch("nr_block_norm_backward", nbytes, dev)
    st = lib.nr_block_norm_backward(packed, index, ws_ptr, nbytes, _stream(index))
    if st:
        raise _nr.NRError("nr_block_norm_backward", st)
    return BlockGrads(dr, du, dgate, *params)


def _flat(t, name, dtype, n, index):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous() or t.get_device() != index or t.data_ptr() % 16:
        raise ValueError(f"{name}: expected a contiguous, 16-byte aligned tensor {dtype} of shape ({n},) on cuda:{index}")
    return t


def _apart(named):
    """Refuses tensors, (name, tensor) each, that share memory."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), i) for i, (_, t) in enumerate(named) if t.numel())
    for (_, end, i), (begin, _, j) in zip(spans, spans[1:]):
        if begin < end:
            raise ValueError(f"{named[min(i, j)][0]} and {named[max(i, j)][0]} overlap")


class AdamWState:
    """What an AdamW step over the tensors `params` keeps (nr_adamw): the averages m
    and v, the step count and, with master, an fp32 master of 16-bit parameters. The
    averages of all tensors lie in one array of `size` values, tensor i's from place
    at[i] on, a multiple of 32. bits 32: m and v are fp32 tensors [size]; bits 8: pairs (codes uint8
    [size], scales uint8 [size / 32]), a quarter of fp32's bytes. master: fp32 [size], the 16-bit
    parameters' values to begin with. step: int64 [1], the steps taken.

    params: contiguous CUDA tensors of one device (fp32, fp16 or bf16), none overlapping
    another or the state's own. m, v, step and a tensor as master are taken as they are, for a state that is
    read back; else they begin with zeros. Every value of the tensors is updated in place. A parameter may move and
    change its dtype between steps, but with master not from fp32 to 16 bits: its master is not kept up while it is fp32."""

    __slots__ = ("params", "bits", "master", "m", "v", "step", "at", "size", "_index", "_shapes", "_device", "_ticket", "_one",
                 "_ws_like", "_table", "_pointers", "_address", "_values", "_types", "_decays")

    def __init__(self, params, bits=32, master=False, m=None, v=None, step=None):
        params = list(params)
        if not params:
            raise ValueError("params: expected at least one tensor")
        if bits not in (32, 8):
            raise ValueError(f"bits: {bits}, expected 32 or 8")
        index = None
        for i, p in enumerate(params):
            name = f"params[{i}]"
            if not isinstance(p, torch.Tensor):
                raise TypeError(f"{name}: expected a torch.Tensor, got {type(p).__name__}")
            if p.dtype not in _DT:
                raise ValueError(f"{name}: dtype {p.dtype}, expected {' or '.join(map(str, _DT))}")
            if not p.is_cuda or (index is not None and p.get_device() != index):
                raise ValueError(f"{name}: expected a tensor on {'a CUDA device' if index is None else f'cuda:{index}'}, "
                                 f"got {p.device}")
            if not p.is_contiguous():
                raise ValueError(f"{name}: must be contiguous")
            index = p.get_device()
        _apart([(f"params[{i}]", p) for i, p in enumerate(params)])
        self.params, self.bits, self._index = params, bits, index
        self.at, size = [], 0
        for p in params:
            self.at.append(size)
            size += -(-p.numel() // _GROUP) * _GROUP
        self.size = size
        dev = params[0].device

        def average(t, name):
            if bits == 32:
                return torch.zeros(size, device=dev) if t is None else _flat(t, name, torch.float32, size, index)
            if t is None:  # zeros: code 0 under the least scale
                return (torch.zeros(size, dtype=torch.uint8, device=dev),
                        torch.full((size // _GROUP,), 12, dtype=torch.uint8, device=dev))
            codes, scales = t
            if not isinstance(scales, torch.Tensor):
                raise TypeError(f"{name}: expected a pair of tensors, codes and scales")
            if scales.dtype != torch.uint8 or scales.shape != (size // _GROUP,) or not scales.is_contiguous() or \
                    scales.get_device() != index:
                raise ValueError(f"{name}: scales: expected a contiguous tensor uint8 of shape ({size // _GROUP},) on cuda:{index}")
            return _flat(codes, name, torch.uint8, size, index), scales

        self.m, self.v = average(m, "m"), average(v, "v")
        self.master = None
        if isinstance(master, torch.Tensor):
            self.master = _flat(master, "master", torch.float32, size, index)
        elif master:
            self.master = torch.zeros(size, device=dev)
            for p, at in zip(params, self.at):
                self.master[at:at + p.numel()] = p.detach().reshape(-1)
        if step is None:
            step = torch.zeros(1, dtype=torch.int64, device=dev)
        elif not isinstance(step, torch.Tensor) or step.dtype != torch.int64 or step.shape != (1,) or step.get_device() != index:
            raise ValueError(f"step: expected a tensor int64 of shape (1,) on cuda:{index}")
        self.step = step
        _apart(self._named())
        self._ticket, self._one = torch.zeros(1, dtype=torch.int32, device=dev), torch.empty(1, device=dev)
        self._shapes, self._device = 2 * [p.shape for p in params], {index}  # of the tensors and gradients
        # what a call passes of them (_TENSOR each, then the values' and the gradients' addresses); the first part is written
        # anew where it changes
        self._pointers = struct.Struct(f"{2 * len(params)}q")
        self._table = bytearray((_TENSOR.size + 16) * len(params))
        self._address = ctypes.addressof((ctypes.c_char * len(self._table)).from_buffer(self._table))
        self._values = self._types = self._decays = self._ws_like = None

    def _named(self):
        """All tensors that a step writes, with their names."""
        out = [(f"params[{i}]", p) for i, p in enumerate(self.params)]
        for name, t in (("m", self.m), ("v", self.v)):
            out += [(name, t)] if self.bits == 32 else [(name, t[0]), (name + "'s scales", t[1])]
        return out + [("step", self.step)] + ([] if self.master is None else [("master", self.master)])

    def _tensors(self):
        out = [*self.params, self.step, self._ticket]
        for t in (self.m, self.v):
            out += [t] if self.bits == 32 else t
        return out if self.master is None else [*out, self.master]

    def _pass(self, grads, decays):
        """Checks the tensors and gradients and writes the table; returns the tensors that have a gradient. A tensor may be
        another one than at the last step (p.data = ...), at the same address too: all that the kernel goes by is looked at
        in every call."""
        count = len(self.params)
        try:  # all of them at once
            every = self.params + grads
            types = [t.dtype for t in every]
            same = types == self._types
            fit = [t.shape for t in every] == self._shapes and set(map(torch.Tensor.get_device, every)) == self._device and \
                all(map(_contiguous, every)) and (same or _DT.keys() >= set(types))
        except (AttributeError, TypeError):  # None, or no tensor
            fit = False
        if fit:
            addresses = list(map(_address, every))
            values = addresses[:count]
        else:
            for i, p in enumerate(self.params):
                if p.dtype not in _DT or p.get_device() != self._index or not p.is_contiguous() or p.shape != self._shapes[i]:
                    raise ValueError(f"params[{i}]: changed to a tensor that the state does not fit")
            addresses, types = _gradients(grads, self._shapes[:count], [self._index] * count)
            values = [p.data_ptr() for p in self.params]
            addresses, types = values + addresses, [p.dtype for p in self.params] + types
            same = types == self._types
        if not same or values != self._values or decays is not self._decays:
            if not same or values != self._values:
                _apart(self._named())
            if self.master is not None and self._types:  # steps in fp32 have left their master as it was
                for i in range(count):
                    if self._types[i] is torch.float32 and types[i] is not torch.float32:
                        raise ValueError(f"params[{i}]: was fp32 in a step before and has no master of these values")
            for i, p in enumerate(self.params):
                _TENSOR.pack_into(self._table, i * _TENSOR.size, p.numel(), self.at[i], _DT[types[i]],
                                  0 if types[count + i] is None else _DT[types[count + i]], decays[i])
            self._values, self._types, self._decays = values, types, decays
        self._pointers.pack_into(self._table, count * _TENSOR.size, *addresses)
        return self.params if fit else [p for p, g in zip(self.params, grads) if g is not None]


def _gradients(grads, shapes, devices):
    """(addresses, types) of gradients, 0 and None for those that are None; checks them."""
    try:  # all of them at once
        types = [g.dtype for g in grads]
        if (shapes is None or [g.shape for g in grads] == shapes) and [g.get_device() for g in grads] == devices and \
                False not in [g.is_contiguous() for g in grads] and _DT.keys() >= set(types):
            return [g.data_ptr() for g in grads], types
    except AttributeError:  # None, or no tensor
        pass
    for i, g in enumerate(grads):
        if g is None:
            continue
        if not isinstance(g, torch.Tensor):
            raise TypeError(f"grads[{i}]: expected a torch.Tensor, got {type(g).__name__}")
        if g.dtype not in _DT or (shapes is not None and g.shape != shapes[i]) or g.get_device() != devices[i] or \
                not g.is_contiguous():
            want = "a contiguous tensor" if shapes is None else f"a contiguous tensor of shape {tuple(shapes[i])}"
            raise ValueError(f"grads[{i}]: {g.dtype} {tuple(g.shape)} on {g.device}, expected {want} in "
                             f"{' or '.join(map(str, _DT))} on cuda:{devices[i]}")
    return [0 if g is None else g.data_ptr() for g in grads], [None if g is None else g.dtype for g in grads]


def _elsewhere_all(fn, stream, tensors, args, kw):
    """_elsewhere for calls on lists of tensors."""
    with torch.cuda.stream(stream):
        out = fn(*args, **kw)
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    return out


def adamw_step(state: AdamWState, grads, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, max_norm=None, seed=0,
               stream=None):
    """One AdamW step of all of the state's tensors (nr_adamw_step), in place: the parameters, the averages,
    the masters and the count. grads: a gradient for each, of its shape, contiguous, in fp32, fp16 or bf16; None
    leaves a tensor as it is. lr: a number, or an fp32 CUDA tensor of one value, which
    a captured step reads anew at every replay. weight_decay: a number, or one for each tensor. max_norm: the
    gradients are scaled so that their common norm is at most that, and the norm, fp32 [1], is
    returned; where it is infinite or NaN nothing is changed, the count neither (its squares are added in
    fp32). seed: of the dither of averages in 8 bits."""
    if not isinstance(state, AdamWState):
        raise TypeError(f"state: expected an AdamWState, got {type(state).__name__}")
    grads = list(grads)
    if stream is not None:
        return _elsewhere_all(adamw_step, stream, [*state._tensors(), *grads, lr], (state, grads, lr),
                              {"betas": betas, "eps": eps, "weight_decay": weight_decay, "max_norm": max_norm, "seed": seed})
    params, index = state.params, state._index
    count = len(params)
    if len(grads) != count:
        raise ValueError(f"grads: {len(grads)}, expected one for each of {count} parameters")
    b1, b2 = betas
    if not (0.0 <= b1 < 1.0 and 0.0 <= b2 < 1.0):
        raise ValueError(f"betas: {betas}, expected two numbers in [0, 1)")
    if not eps > 0.0:
        raise ValueError(f"eps: {eps}, expected a positive number")
    decays = [weight_decay] * count if isinstance(weight_decay, (int, float)) else list(weight_decay)
    if decays == state._decays:
        decays = state._decays
    elif len(decays) != count or not all(0.0 <= d <= _MOST for d in decays):
        raise ValueError("weight_decay: expected a number that is not negative, or one for each parameter")
    lr_at = 0
    if type(lr) is not float and isinstance(lr, torch.Tensor):
        if lr.dtype != torch.float32 or lr.numel() != 1 or lr.get_device() != index:
            raise ValueError(f"lr: expected a number or one fp32 value on cuda:{index}")
        lr_at, lr = lr.data_ptr(), 0.0
    elif not abs(lr) <= _MOST:
        raise ValueError(f"lr: {lr}, expected a finite number of fp32's range")
    if max_norm is not None and not 0.0 < max_norm < float("inf"):
        raise ValueError(f"max_norm: {max_norm}, expected a positive number")
    if not -(1 << 63) <= seed < 1 << 63:
        raise ValueError(f"seed: {seed}, expected a number of 64 bits")
    moved = state._pass(grads, decays)
    first = count * _TENSOR.size
    norm = norm_ptr = ws_ptr = nbytes = 0
    if max_norm is not None:
        norm = torch.empty_like(state._one)  # made the shorter way
        norm_ptr = norm.data_ptr()
    at = state._address
    if state.bits == 32:
        m, v, m_scale, v_scale = state.m.data_ptr(), state.v.data_ptr(), 0, 0
    else:
        (m, m_scale), (v, v_scale) = [[t.data_ptr() for t in pair] for pair in (state.m, state.v)]
    packed = _ADAMW.pack(count, at, at + first, at + first + 8 * count, state.bits,
                         0 if state.master is None else state.master.data_ptr(), m, v, m_scale, v_scale, state.step.data_ptr(),
                         state._ticket.data_ptr(), lr, lr_at, b1, b2, eps, max_norm or 0.0, norm_ptr, seed)
    lib = _nr.lib()
    if norm_ptr:
        if state._ws_like is None:
            state._ws_like, _ = _scratch("nr_adamw_step", lib.nr_adamw_workspace(packed, index), state.step.device)
        ws = torch.empty_like(state._ws_like)  # a call's own, as its stream may be
        ws_ptr, nbytes = ws.data_ptr(), ws.numel()
    st = lib.nr_adamw_step(packed, index, ws_ptr, nbytes, _stream(index))
    if st:
        raise _nr.NRError("nr_adamw_step", st)
    torch.autograd.graph.increment_version(moved)
    return norm if norm_ptr else None


def adamw_read(state: AdamWState, stream=None):
    """The averages (m, v) of a state, [size] each: its own arrays in 32 bits, what the
    codes stand for in 8, exactly, in bf16 (nr_adamw_read)."""
    if not isinstance(state, AdamWState):
        raise TypeError(f"state: expected an AdamWState, got {type(state).__name__}")
    if stream is not None:
        return _elsewhere_all(adamw_read, stream, state._tensors(), (state,), {})
    if state.bits == 32:
        return state.m, state.v
    out = [torch.empty(state.size, dtype=torch.bfloat16, device=state.step.device) for _ in range(2)]
    st = _nr.lib().nr_adamw_read(*[t.data_ptr() for t in (*state.m, *state.v)], state.size, out[0].data_ptr(),
                                 out[1].data_ptr(), state._index, _stream(state._index))
    if st:
        raise _nr.NRError("nr_adamw_read", st)
    return tuple(out)


def grad_norm(grads, stream=None):
    """The 2-norm of all gradients, fp32 [1] on their device (nr_grad_norm). grads: contiguous tensors of one device
    in fp32, fp16 or bf16, None for none."""
    grads = list(grads)
    if stream is not None:
        return _elsewhere_all(grad_norm, stream, grads, (grads,), {})
    first = next((g for g in grads if g is not None), None)
    if first is None:
        raise ValueError("grads: expected at least one tensor")
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        raise (ValueError if isinstance(first, torch.Tensor) else TypeError)("grads: expected CUDA tensors")
    index, dev, count = first.get_device(), first.device, len(grads)
    addresses, types = _gradients(grads, None, [index] * count)
    table = bytearray((_TENSOR.size + 8) * count)
    for i, (g, t) in enumerate(zip(grads, types)):
        if t is not None:
            _TENSOR.pack_into(table, i * _TENSOR.size, g.numel(), 0, 0, _DT[t], 0.0)
    struct.pack_into(f"{count}q", table, count * _TENSOR.size, *addresses)
    hold = (ctypes.c_char * len(table)).from_buffer(table)
    at = ctypes.addressof(hold)
    norm = torch.empty(1, dtype=torch.float32, device=dev)
    packed = _ADAMW.pack(count, at, 0, at + count * _TENSOR.size, 32, 0, 0, 0, 0, 0, 0, 0, 0.0, 0, 0.0, 0.0, 0.0, 0.0, 0, 0)
    lib = _nr.lib()
    nbytes = lib.nr_adamw_workspace(packed, index)
    ws, ws_ptr = _scratch("nr_grad_norm", nbytes, dev)
    st = lib.nr_grad_norm(packed, norm.data_ptr(), index, ws_ptr, nbytes, _stream(index))
    if st:
        raise _nr.NRError("nr_grad_norm", st)
    return norm


def check(device=0):
    """Waits for the device and raises if a bounded wait inside one of these
    operators' kernels expired since the last check (nr_ops_status)."""
    d = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    if d.type != "cuda":
        raise ValueError(f"device: {device}, expected a CUDA device")
    index = torch.cuda.current_device() if d.index is None else d.index
    _nr._check("nr_ops_status", _nr.lib().nr_ops_status(index))

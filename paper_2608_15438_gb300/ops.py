"""Operators for training and serving residual encoders (include/neuroute_ops.h):
the linear layer with its epilogue, the layer norm, their gradients, and
activation checkpoints held in 8 bits.

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

import struct

import torch

from . import neuroute as _nr

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_DT = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_GROUP = 32  # columns that share a checkpoint's scale
_LINEAR = struct.Struct("27q")
_NORM = struct.Struct("4qd17q")


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


def check(device=0):
    """Waits for the device and raises if a bounded wait inside one of these
    operators' kernels expired since the last check (nr_ops_status)."""
    d = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    if d.type != "cuda":
        raise ValueError(f"device: {device}, expected a CUDA device")
    index = torch.cuda.current_device() if d.index is None else d.index
    _nr._check("nr_ops_status", _nr.lib().nr_ops_status(index))

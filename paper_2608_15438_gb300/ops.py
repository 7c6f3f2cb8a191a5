"""Operators for training and serving residual encoders (include/neuroute_ops.h):
the linear layer with its epilogue, the layer norm, their gradients, and
activation checkpoints held in 8 bits.

Argument checks and marshalling only; every step runs in the library's
kernels and there is no fallback. Matrices are CUDA tensors of two dimensions
with any row pitch (stride(1) == 1); a wrong tensor raises before any call.
Work goes to the current stream of the tensors' device, or to `stream`, on
which the outputs are then allocated. Nothing synchronises.
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
        self.codes, self.scales, self.shape, self.dtype = codes, scales, tuple(shape), dtype

    @property
    def device(self):
        return self.codes.device

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()

    def record_stream(self, stream):
        self.codes.record_stream(stream)
        self.scales.record_stream(stream)


def _matrix(t, name, dtypes, rows, cols, device):
    """Checks a row-major matrix; returns its row pitch in elements."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    sh = t.shape
    if len(sh) != 2 or (rows is not None and sh[0] != rows) or (cols is not None and sh[1] != cols):
        raise ValueError(f"{name}: shape {tuple(sh)}, expected ({'any' if rows is None else rows}, "
                         f"{'any' if cols is None else cols})")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name}: expected a tensor on {device or 'a CUDA device'}, got {t.device}")
    ld, inner = t.stride()
    if inner != 1 and sh[1] > 1:
        raise ValueError(f"{name}: rows must be contiguous (stride(1) == 1)")
    return ld


def _vector(t, name, dtypes, n, device):
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.shape != (n,):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({n},)")
    if t.device != device:
        raise ValueError(f"{name}: expected a tensor on {device}, got {t.device}")
    if n > 1 and t.stride(0) != 1:
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _held(c, name, rows, cols, device, dtype):
    if (rows is not None and c.shape[0] != rows) or (cols is not None and c.shape[1] != cols):
        raise ValueError(f"{name}: shape {c.shape}, expected ({'any' if rows is None else rows}, "
                         f"{'any' if cols is None else cols})")
    if device is not None and c.device != device:
        raise ValueError(f"{name}: expected a checkpoint on {device}, got {c.device}")
    if dtype is not None and c.dtype != dtype:
        raise ValueError(f"{name}: made from {c.dtype}, expected {dtype}")


def _act(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"act: {name!r}, expected one of {', '.join(ACTIVATIONS)}") from None


def _widths(*dims):
    for d in dims:
        if d < 1 or d >= 1 << 24:
            raise ValueError(f"widths from 1 to 2^24 - 1 are supported, got {d}")


def _raw(device):
    return torch.cuda.current_stream(device).cuda_stream


def _elsewhere(fn, stream, args, kw):
    """fn on another stream: outputs and scratch belong to it, inputs stay alive for it."""
    with torch.cuda.stream(stream):
        out = fn(*args, **kw)
    for t in list(args) + list(kw.values()):
        if isinstance(t, Checkpoint8) or (isinstance(t, torch.Tensor) and t.is_cuda):
            t.record_stream(stream)
    return out


def _run(call, packed, index, device, ws_bytes):
    if ws_bytes < 0:
        raise _nr.NRError(call, -1)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=device) if ws_bytes else None
    st = getattr(_nr.lib(), call)(packed, index, ws.data_ptr() if ws_bytes else 0, ws_bytes, _raw(device))
    if st:
        raise _nr.NRError(call, st)


def _new_checkpoint(m, n, dtype, device):
    g = -(-n // _GROUP)
    return Checkpoint8(torch.empty((m, g * _GROUP), dtype=torch.int8, device=device),
                       torch.empty((m, g), dtype=torch.uint8, device=device), (m, n), dtype)


def checkpoint8(x, stream=None) -> Checkpoint8:
    """x [m x n] (fp32, fp16 or bf16) held in 8 bits (nr_checkpoint8_write)."""
    if stream is not None:
        return _elsewhere(checkpoint8, stream, (x,), {})
    ld = _matrix(x, "x", tuple(_DT), None, None, None)
    m, n = x.shape
    _widths(n)
    c = _new_checkpoint(m, n, x.dtype, x.device)
    st = _nr.lib().nr_checkpoint8_write(x.data_ptr(), _DT[x.dtype], m, n, ld, c.codes.data_ptr(),
                                        c.scales.data_ptr(), x.device.index, _raw(x.device))
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
    st = _nr.lib().nr_checkpoint8_read(c.codes.data_ptr(), c.scales.data_ptr(), m, n, a, y.data_ptr(),
                                       _DT[c.dtype], n, c.device.index, _raw(c.device))
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
    x_ld = _matrix(x, "x", (torch.float16, torch.bfloat16), None, None, None)
    m, k = x.shape
    dt, dev = x.dtype, x.device
    w_ld = _matrix(w, "w", (dt,), None, k, dev)
    n = w.shape[0]
    _widths(k, n)
    b = _vector(bias, "bias", (dt, torch.float32), n, dev)
    a = _act(act)
    r = r_ld = 0
    if residual is not None:
        r_ld, r = _matrix(residual, "residual", (dt,), m, n, dev), residual.data_ptr()
    ydt = dt if out_dtype is None else out_dtype
    if ydt is not dt and ydt is not torch.float32:
        raise ValueError(f"out_dtype: {out_dtype}, expected {dt} or torch.float32")
    y = torch.empty((m, n), dtype=ydt, device=dev)
    z = zp = zs = None
    if save == "z":
        z = torch.empty((m, n), dtype=dt, device=dev)
        zp = z.data_ptr()
    elif save == "z8":
        z = _new_checkpoint(m, n, dt, dev)
        zp, zs = z.codes.data_ptr(), z.scales.data_ptr()
    elif save is not None:
        raise ValueError(f"save: {save!r}, expected None, 'z' or 'z8'")
    code = _DT[dt]
    packed = _LINEAR.pack(m, k, n, code, _DT[ydt], code if bias is None else _DT[bias.dtype], a, x.data_ptr(),
                          x_ld, 0, 0, w.data_ptr(), w_ld, b, r, r_ld, y.data_ptr(), n, zp or 0, n, zs or 0,
                          0, 0, 0, 0, 0, 0)
    _run("nr_linear_forward", packed, dev.index, dev,
         _nr.lib().nr_linear_forward_workspace(packed, dev.index) if m else 0)
    return y if z is None else (y, z)


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
    w_ld = _matrix(w, "w", (torch.float16, torch.bfloat16), None, None, None)
    n, k = w.shape
    _widths(k, n)
    dt, dev = w.dtype, w.device
    dy_ld = _matrix(dy, "dy", (dt, torch.float32), None, n, dev)
    m = dy.shape[0]
    xs = zp = z_ld = zs = 0
    if isinstance(x, Checkpoint8):
        _held(x, "x", m, k, dev, dt)
        xp, x_ld, xs = x.codes.data_ptr(), 0, x.scales.data_ptr()
    else:
        x_ld, xp = _matrix(x, "x", (dt,), m, k, dev), x.data_ptr()
        if x_act != "none":
            raise ValueError("x_act: only for an x held in 8 bits")
    a, xa = _act(act), _act(x_act)
    if a:
        if z is None:
            raise ValueError("z: needed with an activation (linear's save='z' or 'z8')")
        if isinstance(z, Checkpoint8):
            _held(z, "z", m, n, dev, dt)
            zp, zs = z.codes.data_ptr(), z.scales.data_ptr()
        else:
            z_ld, zp = _matrix(z, "z", (dt,), m, n, dev), z.data_ptr()
    bdt = torch.float32 if bias_dtype is None else bias_dtype
    if bdt is not dt and bdt is not torch.float32:
        raise ValueError(f"bias_dtype: {bias_dtype}, expected {dt} or torch.float32")
    dx = torch.empty((m, k), dtype=dt, device=dev) if need[0] else None
    dw = torch.empty((n, k), dtype=dt, device=dev) if need[1] else None
    db = torch.empty(n, dtype=bdt, device=dev) if need[2] else None
    packed = _LINEAR.pack(m, k, n, _DT[dt], _DT[dy.dtype], _DT[bdt], a, xp, x_ld, xs, xa, w.data_ptr(), w_ld,
                          0, 0, 0, 0, 0, zp, z_ld, zs, dy.data_ptr(), dy_ld,
                          dx.data_ptr() if need[0] else 0, k, dw.data_ptr() if need[1] else 0,
                          db.data_ptr() if need[2] else 0)
    _run("nr_linear_backward", packed, dev.index, dev,
         _nr.lib().nr_linear_backward_workspace(packed, dev.index) if m else 0)
    return dx, dw, db


def layer_norm(x, weight=None, bias=None, eps=1e-5, save=False, stream=None):
    """y = (x - mean) rstd weight + bias over the rows of x [m x n]
    (nr_layer_norm_forward), in x's dtype (fp32, fp16 or bf16; a Checkpoint8:
    the one it was made from); weight and bias [n] in that dtype or fp32, both
    the same. save: returns (y, mean, rstd), mean and rstd [m] fp32."""
    if stream is not None:
        return _elsewhere(layer_norm, stream, (x, weight, bias), {"eps": eps, "save": save})
    xs = x_ld = 0
    if isinstance(x, Checkpoint8):
        xp, xs = x.codes.data_ptr(), x.scales.data_ptr()
    else:
        x_ld, xp = _matrix(x, "x", tuple(_DT), None, None, None), x.data_ptr()
    m, n = x.shape
    dt, dev = x.dtype, x.device
    _widths(n)
    wdt = weight.dtype if isinstance(weight, torch.Tensor) else bias.dtype if isinstance(bias, torch.Tensor) else dt
    w = _vector(weight, "weight", (dt, torch.float32), n, dev)
    b = _vector(bias, "bias", (wdt,) if weight is not None else (dt, torch.float32), n, dev)
    if not eps > 0.0:
        raise ValueError(f"eps: {eps}, expected a positive number")
    y = torch.empty((m, n), dtype=dt, device=dev)
    mean = rstd = None
    if save:
        mean = torch.empty(m, dtype=torch.float32, device=dev)
        rstd = torch.empty(m, dtype=torch.float32, device=dev)
    packed = _NORM.pack(m, n, _DT[dt], _DT[wdt], eps, xp, x_ld, xs, w, b, y.data_ptr(), n,
                        mean.data_ptr() if save else 0, rstd.data_ptr() if save else 0, 0, 0, 0, 0, 0, 0, 0, 0)
    st = _nr.lib().nr_layer_norm_forward(packed, dev.index, _raw(dev))
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
    dy_ld = _matrix(dy, "dy", tuple(_DT), None, None, None)
    m, n = dy.shape
    dt, dev = dy.dtype, dy.device
    _widths(n)
    xs = x_ld = r = r_ld = 0
    if isinstance(x, Checkpoint8):
        _held(x, "x", m, n, dev, dt)
        xp, xs = x.codes.data_ptr(), x.scales.data_ptr()
    else:
        x_ld, xp = _matrix(x, "x", (dt,), m, n, dev), x.data_ptr()
    w = _vector(weight, "weight", (dt, torch.float32), n, dev)
    mp = _vector(mean, "mean", (torch.float32,), m, dev)
    rp = _vector(rstd, "rstd", (torch.float32,), m, dev)
    if mean is None or rstd is None:
        raise ValueError("mean, rstd: needed (layer_norm's save=True)")
    if residual_grad is not None:
        r_ld, r = _matrix(residual_grad, "residual_grad", (dt,), m, n, dev), residual_grad.data_ptr()
    wdt = torch.float32 if weight is None else weight.dtype
    dx = torch.empty((m, n), dtype=dt, device=dev)
    dw = db = None
    if param_grads:
        dw = torch.empty(n, dtype=wdt, device=dev)
        db = torch.empty(n, dtype=wdt, device=dev)
    packed = _NORM.pack(m, n, _DT[dt], _DT[wdt], 0.0, xp, x_ld, xs, w, 0, 0, 0, mp, rp, dy.data_ptr(), dy_ld, r,
                        r_ld, dx.data_ptr(), n, dw.data_ptr() if param_grads else 0,
                        db.data_ptr() if param_grads else 0)
    _run("nr_layer_norm_backward", packed, dev.index, dev,
         _nr.lib().nr_layer_norm_backward_workspace(packed, dev.index) if m else 0)
    return dx, dw, db


def check(device=0):
    """Waits for the device and raises if a bounded wait inside one of these
    operators' kernels expired since the last check (nr_ops_status)."""
    _nr._check("nr_ops_status", _nr.lib().nr_ops_status(torch.device("cuda", device).index
                                                         if isinstance(device, int) else device.index))

"""What stands around a long convolution in a layer: norm, 8-bit projections, activations kept in 8 bits (see include/fftconv.h, "The layers
around a convolution").

    rows, h, rstd = layers.rms_norm_i8(x, weight, residual=r)                  # (b, n, d): h = x + r, its norm in 8 bits
    u, w, v = layers.linear_i8(rows, in_proj, layout="channels", parts=3)      # three of (b, h, n), what Plan.forward_gated takes
    y = plan.forward_gated(u, w, v, kf)

Argument marshalling only, as in fftconv.py: every step runs in the HIP kernels of the library, on the current stream of the current
device; PyTorch supplies memory. Tensors that are not laid out as a call wants them are refused, not copied.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import fftconv as _f

RUN = 128       # samples of a channel that share a scale in a checkpoint
MAX_ROW = 16384


class Rows8(NamedTuple):
    """Rows in 8 bits: q (..., d) int8 and a scale for each row, (...) fp32; row i stands for q[i] * scale[i]."""
    q: torch.Tensor
    scale: torch.Tensor

    def float(self):
        return self.q * self.scale[..., None]


class Checkpoint8(NamedTuple):
    """Activations in 8 bits: q (b, c, n) int8 and scale (b, c, ceil(n / 128)) fp32, one for 128 samples of a channel."""
    q: torch.Tensor
    scale: torch.Tensor


def _on_gpu(name, t, dtypes, dim=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or (dim is not None and t.dim() != dim):
        raise ValueError("%s must be a CUDA tensor%s of %s" % (name, "" if dim is None else " of %d dimensions" % dim,
                                                               " / ".join(str(d).replace("torch.", "") for d in dtypes)))
    if t.device.index != _f._current_device():
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    return t


_IO = tuple(_f._DTYPE_CODE)
_F32, _I8 = (torch.float32,), (torch.int8,)


def _contiguous(name, t, dtypes, dim=None, shape=None):
    _on_gpu(name, t, dtypes, dim)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have the shape %s" % (name, tuple(shape)))
    return t


def _rows(name, x, dtypes=_IO):
    """(rows, values of a row, distance between rows) of x (..., d): contiguous values, rows at one distance (a slice of wider rows will do)."""
    _on_gpu(name, x, dtypes)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("%s must have rows of one value at least" % name)
    d = x.shape[-1]
    if x.is_contiguous():
        return x.numel() // d, d, d
    ld, t = None, 1
    for size, stride in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = stride
        elif stride != ld * t:
            ld = -1
            break
        t *= size
    ld = d if ld is None else ld
    if (x.stride(-1) != 1 and d > 1) or ld < d:
        raise ValueError("%s must have contiguous values and rows at one distance" % name)
    return x.numel() // d, d, ld


def _ptr(t):
    return None if t is None else t.data_ptr()


def _weight(weight, d):
    return _contiguous("weight", weight, _F32, 1, (d,))


def _norm(x, weight, residual, eps, i8):
    t, d, ldx = _rows("x", x)
    _weight(weight, d)
    ldr = 0
    if residual is not None:
        _, _, ldr = _rows("residual", residual, (x.dtype,))
        if residual.shape != x.shape:
            raise ValueError("x and residual differ in shape")
    y = torch.empty(x.shape, dtype=torch.int8 if i8 else x.dtype, device=x.device)
    h = x if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if i8 else None
    rc = _f.load().fftconv_rms_norm(x.data_ptr(), ldx, _ptr(residual), ldr, weight.data_ptr(), y.data_ptr(), None if residual is None else h.data_ptr(),
                                    rstd.data_ptr(), _ptr(scale), t, d, eps, _f._DTYPE_CODE[x.dtype], _f._stream_ptr())
    if rc:
        _f._check(rc)
    return (Rows8(y, scale) if i8 else y), h, rstd


def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """fftconv_rms_norm: (y, h, rstd) with h = x + residual (x itself without one) and y = h * rstd * weight, rstd = 1 / sqrt(mean(h^2) + eps).
    x, residual: (..., d) fp32, fp16 or bf16; weight: (d,) fp32. h and rstd are what rms_norm_backward takes."""
    return _norm(x, weight, residual, eps, False)


def rms_norm_i8(x, weight, residual=None, eps: float = 1e-6):
    """As rms_norm, with y in 8 bits and a scale for each row (Rows8), what linear_i8 takes."""
    return _norm(x, weight, residual, eps, True)


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    """fftconv_rms_norm_backward: (dx, dweight); dx is the gradient of x and of the residual alike, dh what comes back along the residual
    stream (None: nothing), dweight fp32."""
    t, d, lddy = _rows("dy", dy)
    _weight(weight, d)
    _contiguous("h", h, (dy.dtype,), None, dy.shape)
    _contiguous("rstd", rstd, _F32, None, dy.shape[:-1])
    if dh is not None:
        _contiguous("dh", dh, (dy.dtype,), None, dy.shape)
    lib, code = _f.load(), _f._DTYPE_CODE[dy.dtype]
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
    if t == 0:
        return dx, torch.zeros(d, dtype=torch.float32, device=dy.device)
    dw = torch.empty(d, dtype=torch.float32, device=dy.device)
    ws = torch.empty(lib.fftconv_workspace_bytes_rms_norm_backward(t, d, code), dtype=torch.uint8, device=dy.device)
    rc = lib.fftconv_rms_norm_backward(dy.data_ptr(), lddy, h.data_ptr(), _ptr(dh), weight.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(),
                                       t, d, code, ws.data_ptr(), _f._stream_ptr())
    if rc:
        _f._check(rc)
    return dx, dw


def quantize_rows(x):
    """fftconv_quantize_rows: x (..., d) in 8 bits with a scale for each row (Rows8); a projection's weight (o, k) for linear_i8, once."""
    t, d, ldx = _rows("x", x)
    q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rc = _f.load().fftconv_quantize_rows(x.data_ptr(), ldx, q.data_ptr(), scale.data_ptr(), t, d, _f._DTYPE_CODE[x.dtype], _f._stream_ptr())
    if rc:
        _f._check(rc)
    return Rows8(q, scale)


def linear_i8(rows, weight, bias=None, dtype=torch.bfloat16, layout: str = "tokens", parts: int = 1):
    """fftconv_linear_i8: rows (b, n, k) (or (t, k): one sequence) and weight (o, k), both Rows8 or pairs (q, scale); bias (o,) fp32.
    layout "tokens": y (b, n, o). "channels": y (b, o, n), or (parts, b, o / parts, n) with parts > 1."""
    (xq, xs), (wq, ws) = rows, weight
    _contiguous("rows", xq, _I8)
    if xq.dim() not in (2, 3):
        raise ValueError("rows must be (b, n, k) or (t, k)")
    _contiguous("the rows' scale", xs, _F32, None, xq.shape[:-1])
    _contiguous("weight", wq, _I8, 2)
    o, k = wq.shape
    _contiguous("the weight's scale", ws, _F32, None, (o,))
    if xq.shape[-1] != k:
        raise ValueError("rows and weight differ in length")
    if bias is not None:
        _contiguous("bias", bias, _F32, 1, (o,))
    if dtype not in _f._DTYPE_CODE:
        raise ValueError("dtype must be fp32, fp16 or bf16")
    parts = int(parts)
    if layout not in ("tokens", "channels") or parts < 1 or (layout == "tokens" and parts != 1) or o % parts:
        raise ValueError("layout is \"tokens\" or \"channels\", parts a divisor of the output channels (1 for tokens)")
    b, n = (1, xq.shape[0]) if xq.dim() == 2 else xq.shape[:2]
    if layout == "tokens":
        shape = (*xq.shape[:-1], o)
    else:
        shape = (parts, b, o // parts, n) if parts > 1 else (b, o, n)
        shape = shape if xq.dim() == 3 else shape[:-3] + shape[-2:]
    y = torch.empty(shape, dtype=dtype, device=xq.device)
    if y.numel() == 0:
        return y
    p, code, lib = 0 if layout == "tokens" else parts, _f._DTYPE_CODE[dtype], _f.load()
    need = lib.fftconv_workspace_bytes_linear_i8(b, n, k, o, p, code)
    work = torch.empty(need, dtype=torch.uint8, device=xq.device) if need else None
    rc = lib.fftconv_linear_i8(xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), _ptr(bias), y.data_ptr(), b, n, k, o, p, code, _ptr(work),
                               _f._stream_ptr())
    if rc:
        _f._check(rc)
    return y


def act_pack(x, layout: str = "channels"):
    """fftconv_act_pack: x (b, c, n), or (b, n, c) with layout "tokens", in 8 bits (Checkpoint8, channel by channel either way)."""
    _contiguous("x", x, _IO, 3)
    if layout not in ("tokens", "channels"):
        raise ValueError("layout is \"tokens\" or \"channels\"")
    b, c, n = x.shape if layout == "channels" else (x.shape[0], x.shape[2], x.shape[1])
    q = torch.empty((b, c, n), dtype=torch.int8, device=x.device)
    scale = torch.empty((b, c, -(-n // RUN)), dtype=torch.float32, device=x.device)
    if q.numel():
        rc = _f.load().fftconv_act_pack(x.data_ptr(), q.data_ptr(), scale.data_ptr(), b, c, n, layout == "tokens", _f._DTYPE_CODE[x.dtype], _f._stream_ptr())
        if rc:
            _f._check(rc)
    return Checkpoint8(q, scale)


def _kept(name, p):
    q, scale = p
    _contiguous(name, q, _I8, 3)
    _contiguous("the scale of " + name, scale, _F32, 3, (*q.shape[:2], -(-q.shape[2] // RUN)))
    return q, scale


def act_unpack(p, dtype=torch.bfloat16, gate=None):
    """fftconv_act_unpack: the activations of a Checkpoint8 (or a pair (q, scale)), (b, c, n) in dtype; times `gate`, a second one or a tensor in
    dtype, with one rounding."""
    q, scale = _kept("the checkpoint", p)
    if dtype not in _f._DTYPE_CODE:
        raise ValueError("dtype must be fp32, fp16 or bf16")
    gq = gs = gt = None
    if isinstance(gate, torch.Tensor):
        gt = _contiguous("gate", gate, (dtype,), 3, q.shape)
    elif gate is not None:
        gq, gs = _kept("gate", gate)
        if gq.shape != q.shape:
            raise ValueError("the checkpoint and its gate differ in shape")
    x = torch.empty(q.shape, dtype=dtype, device=q.device)
    if x.numel():
        b, c, n = q.shape
        rc = _f.load().fftconv_act_unpack(q.data_ptr(), scale.data_ptr(), _ptr(gq), _ptr(gs), _ptr(gt), x.data_ptr(), b, c, n, _f._DTYPE_CODE[dtype],
                                          _f._stream_ptr())
        if rc:
            _f._check(rc)
    return x


def linear_grad_weight(dy, p, layout: str = "tokens", dtype=torch.float32):
    """fftconv_linear_grad_weight: the gradient (o, c) of a projection's weight from dy, (b, n, o) or with layout "channels" (b, o, n), and
    the projection's input kept in 8 bits (Checkpoint8 of (b, c, n)). dtype: fp32 or that of dy."""
    q, scale = _kept("the checkpoint", p)
    _contiguous("dy", dy, _IO, 3)
    if layout not in ("tokens", "channels"):
        raise ValueError("layout is \"tokens\" or \"channels\"")
    if dtype not in (torch.float32, dy.dtype):
        raise ValueError("dtype must be fp32 or that of dy")
    b, c, n = q.shape
    o = dy.shape[2] if layout == "tokens" else dy.shape[1]
    if tuple(dy.shape) != ((b, n, o) if layout == "tokens" else (b, o, n)):
        raise ValueError("dy and the checkpoint differ in sequences or samples")
    if not b * n * c * o:
        return torch.zeros((o, c), dtype=dtype, device=dy.device)
    lib, code, tokens = _f.load(), _f._DTYPE_CODE[dy.dtype], layout == "tokens"
    dw = torch.empty((o, c), dtype=dtype, device=dy.device)
    ws = torch.empty(lib.fftconv_workspace_bytes_linear_grad_weight(b, n, o, c, tokens, code), dtype=torch.uint8, device=dy.device)
    rc = lib.fftconv_linear_grad_weight(dy.data_ptr(), q.data_ptr(), scale.data_ptr(), dw.data_ptr(), b, n, o, c, tokens, code, _f._DTYPE_CODE[dtype],
                                        ws.data_ptr(), _f._stream_ptr())
    if rc:
        _f._check(rc)
    return dw

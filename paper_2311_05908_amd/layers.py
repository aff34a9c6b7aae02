"""What stands around a long convolution in a layer: norm, 8-bit projections, activations kept in 8 bits (see include/fftconv.h, "The layers
around a convolution").

    rows, h, rstd = layers.rms_norm_i8(x, weight, residual=r)                  # (b, n, d): h = x + r, its norm in 8 bits
    u, w, v = layers.linear_i8(rows, in_proj, layout="channels", parts=3)      # three of (b, h, n), what Plan.forward_gated takes
    y = plan.forward_gated(u, w, v, kf)

Argument marshalling only, as in fftconv.py: every step runs in the HIP kernels of the library, on the current stream of the current
device; PyTorch supplies memory. Tensors that are not laid out as a call wants them are refused, not copied.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from . import fftconv as _f

RUN = 128       # samples of a channel that share a scale in a checkpoint


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


_IO = tuple(_f._DTYPE_CODE)
_F32, _I8 = (torch.float32,), (torch.int8,)
_CODE = _f._DTYPE_CODE
_device = _f._current_device
_empty = torch.empty


def _refuse(name, t, dtypes, dim, shape):
    """Why _contiguous does not take t."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or (dim is not None and t.dim() != dim):
        raise ValueError("%s must be a CUDA tensor%s of %s" % (name, "" if dim is None else " of %d dimensions" % dim,
                                                               " / ".join(str(d).replace("torch.", "") for d in dtypes)))
    if t.get_device() != _device():
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have the shape %s" % (name, tuple(shape)))
    raise ValueError("%s must be contiguous" % name)


def _contiguous(name, t, dtypes, dim=None, shape=None):
    """t, if it is on the current device, contiguous, and of one of the types, with so many dimensions or that shape. (A CPU tensor's device is -1.)"""
    if (not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not t.is_contiguous() or not t.is_cuda or t.get_device() != _device()
            or (dim is not None and t.dim() != dim) or (shape is not None and t.shape != shape)):
        _refuse(name, t, dtypes, dim, shape)
    return t


def _rows(name, x, dtypes=_IO):
    """(rows, values of a row, distance between rows) of x (..., d): contiguous values, rows at one distance (a slice of wider rows will do)."""
    if not isinstance(x, torch.Tensor) or x.dtype not in dtypes or not x.is_cuda or x.get_device() != _device():
        _refuse(name, x, dtypes, None, None)
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError("%s must have rows of one value at least" % name)
    d = shape[-1]
    if x.is_contiguous():
        return x.numel() // d, d, d
    ld, t = None, 1
    for size, stride in zip(reversed(shape[:-1]), reversed(x.stride()[:-1])):
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


@functools.lru_cache(maxsize=None)
def _calls(lib):
    """The entry points of a library as functions of integers, addresses and None, through the binding's extension where it can be built."""
    fast = _f._fastcall()
    c = {name: _f._entry(lib, "fftconv_" + name) for name in ("rms_norm_backward", "linear_i8", "act_pack", "act_unpack", "linear_grad_weight")}
    c["quantize_rows"] = lib.fftconv_quantize_rows
    if fast is None:
        c["rms_norm"] = lambda eps, *a: lib.fftconv_rms_norm(*a[:11], eps, *a[11:])
    else:
        c["rms_norm"] = functools.partial(_f._extension().call_norm, ctypes.cast(lib.fftconv_rms_norm, ctypes.c_void_p).value)
    return type("Calls", (), {k: staticmethod(v) for k, v in c.items()})


@functools.lru_cache(maxsize=1024)
def _workspace(lib, name, *sizes):
    """Bytes of workspace, a function of the sizes."""
    return int(getattr(lib, "fftconv_workspace_bytes_" + name)(*sizes))


def _norm(x, weight, residual, eps, i8):
    t, d, ldx = _rows("x", x)
    _contiguous("weight", weight, _F32, 1, (d,))
    shape, dtype, device = x.shape, x.dtype, x.device
    rows = shape[:-1]
    rp, ldr = None, 0
    if residual is not None:
        if not isinstance(residual, torch.Tensor) or residual.shape != shape or residual.dtype != dtype:
            raise ValueError("residual must be a tensor of the shape and type of x")
        _, _, ldr = _rows("residual", residual)
        rp = residual.data_ptr()
    if residual is None and x.is_contiguous():
        h, hp = x, None
    else:
        # (empty_like: 1.2 us where empty takes 2.1, of the 13 that a call on one row takes)
        h = torch.empty_like(x, memory_format=torch.contiguous_format) if ldx == d else _empty(shape, dtype=dtype, device=device)
        hp = h.data_ptr()
    y = torch.empty_like(x, dtype=torch.int8 if i8 else dtype, memory_format=torch.contiguous_format) if ldx == d else _empty(shape, dtype=torch.int8 if i8 else dtype, device=device)
    if i8:
        rstd, scale = _empty(rows, dtype=torch.float32, device=device), _empty(rows, dtype=torch.float32, device=device)
        sp = scale.data_ptr()
    else:
        rstd, sp = _empty(rows, dtype=torch.float32, device=device), None
    rc = _calls(_f.load()).rms_norm(eps, x.data_ptr(), ldx, rp, ldr, weight.data_ptr(), y.data_ptr(), hp, rstd.data_ptr(), sp, t, d, _CODE[dtype],
                                    _f._stream_ptr())
    if rc:
        _f._check(rc)
    return (Rows8(y, scale) if i8 else y), h, rstd


def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """fftconv_rms_norm: (y, h, rstd) with h = x + residual and y = h * rstd * weight, rstd = 1 / sqrt(mean(h^2) + eps).
    x, residual: (..., d) fp32, fp16 or bf16; weight: (d,) fp32. h and rstd are what rms_norm_backward takes. Without a residual h is x itself where x
    is contiguous (what is written into x before the backward pass is then in h too), else a contiguous copy."""
    return _norm(x, weight, residual, eps, False)


def rms_norm_i8(x, weight, residual=None, eps: float = 1e-6):
    """As rms_norm, with y in 8 bits and a scale for each row (Rows8), what linear_i8 takes."""
    return _norm(x, weight, residual, eps, True)


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    """fftconv_rms_norm_backward: (dx, dweight); dx is the gradient of x and of the residual alike, dh what comes back along the residual
    stream (None: nothing), dweight fp32."""
    t, d, lddy = _rows("dy", dy)
    _contiguous("weight", weight, _F32, 1, (d,))
    shape, dtype = dy.shape, dy.dtype
    _contiguous("h", h, (dtype,), None, shape)
    _contiguous("rstd", rstd, _F32, None, shape[:-1])
    if dh is not None:
        _contiguous("dh", dh, (dtype,), None, shape)
    lib, code = _f.load(), _CODE[dtype]
    dx = _empty(shape, dtype=dtype, device=dy.device)
    if t == 0:
        return dx, torch.zeros(d, dtype=torch.float32, device=dy.device)
    dw = _empty(d, dtype=torch.float32, device=dy.device)
    need = _workspace(lib, "rms_norm_backward", t, d, code)
    ws = _empty(need, dtype=torch.uint8, device=dy.device) if need else None
    rc = _calls(lib).rms_norm_backward(dy.data_ptr(), lddy, h.data_ptr(), _ptr(dh), weight.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(),
                                       t, d, code, _ptr(ws), _f._stream_ptr())
    if rc:
        _f._check(rc)
    return dx, dw


def quantize_rows(x):
    """fftconv_quantize_rows: x (..., d) in 8 bits with a scale for each row (Rows8); a projection's weight (o, k) for linear_i8, once."""
    t, d, ldx = _rows("x", x)
    q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rc = _calls(_f.load()).quantize_rows(x.data_ptr(), ldx, q.data_ptr(), scale.data_ptr(), t, d, _f._DTYPE_CODE[x.dtype], _f._stream_ptr())
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
    need = _workspace(lib, "linear_i8", b, n, k, o, p, code)
    work = torch.empty(need, dtype=torch.uint8, device=xq.device) if need else None
    rc = _calls(lib).linear_i8(xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), _ptr(bias), y.data_ptr(), b, n, k, o, p, code, _ptr(work),
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
        rc = _calls(_f.load()).act_pack(x.data_ptr(), q.data_ptr(), scale.data_ptr(), b, c, n, int(layout == "tokens"), _CODE[x.dtype], _f._stream_ptr())
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
    dtype, the product in fp32."""
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
        rc = _calls(_f.load()).act_unpack(q.data_ptr(), scale.data_ptr(), _ptr(gq), _ptr(gs), _ptr(gt), x.data_ptr(), b, c, n, _f._DTYPE_CODE[dtype],
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
    lib, code, tokens = _f.load(), _CODE[dy.dtype], int(layout == "tokens")
    dw = torch.empty((o, c), dtype=dtype, device=dy.device)
    ws = torch.empty(_workspace(lib, "linear_grad_weight", b, n, o, c, tokens, code), dtype=torch.uint8, device=dy.device)
    rc = _calls(lib).linear_grad_weight(dy.data_ptr(), q.data_ptr(), scale.data_ptr(), dw.data_ptr(), b, n, o, c, tokens, code, _f._DTYPE_CODE[dtype],
                                        ws.data_ptr(), _f._stream_ptr())
    if rc:
        _f._check(rc)
    return dw

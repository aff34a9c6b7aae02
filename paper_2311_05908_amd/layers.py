"""What stands around a long convolution in a layer: norm, 8-bit projections, activations kept in 8 bits; a gated recurrence for its place; clipping of
gradients (see include/fftconv.h, from "The layers around a convolution" on).

    rows, h, rstd = layers.rms_norm_i8(x, weight, residual=r)                  # (b, n, d): h = x + r, its norm in 8 bits
    u, w, v = layers.linear_i8(rows, in_proj, layout="channels", parts=3)      # three of (b, h, n), what Plan.forward_gated takes
    y = plan.forward_gated(u, w, v, kf)
    y, state = layers.gated_scan(u, w, v=v)                                    # or a recurrence, and its state

Argument marshalling only, as in fftconv.py: every step runs in the HIP kernels of the library, on the current stream of the current
device; PyTorch supplies memory. Tensors that are not laid out as a call wants them are refused, not copied.
"""
from __future__ import annotations

import array
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


class Blocks8(NamedTuple):
    """Rows in 8-bit floating point: q (..., k) e4m3 and scale (ceil(k / 128), ...) fp32, block by block: scale[j, i] is that of q[i, 128 j : 128 (j + 1)]."""
    q: torch.Tensor
    scale: torch.Tensor

    def float(self):
        k = self.q.shape[-1]
        return self.q.float() * self.scale.movedim(0, -1).repeat_interleave(128, -1)[..., :k]


class Tiles8(NamedTuple):
    """A weight in 8-bit floating point: q (o, k) e4m3 and scale (ceil(o / 128), ceil(k / 128)) fp32, one for 128 x 128."""
    q: torch.Tensor
    scale: torch.Tensor

    def float(self):
        o, k = self.q.shape
        return self.q.float() * self.scale.repeat_interleave(128, 0)[:o].repeat_interleave(128, 1)[:, :k]


_IO = tuple(_f._DTYPE_CODE)
_F8 = torch.float8_e4m3fn
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
    c = {name: _f._entry(lib, "fftconv_" + name) for name in ("rms_norm_backward", "linear_i8", "act_pack", "act_unpack", "linear_grad_weight",
                                                             "gated_scan", "gated_scan_backward", "gated_step", "quantize_blocks_channels",
                                                             "quantize_tiles", "linear_f8")}
    c["quantize_rows"], c["quantize_blocks"] = lib.fftconv_quantize_rows, lib.fftconv_quantize_blocks
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


_GATES = {"sigmoid": 0, "log": 1}


def _scanned(u, w, v, lengths, gate):
    """(b, c, n), dtype, code and gate of a scan's operands. (All checks together; what does not pass is gone through once more for what is wrong with it.)"""
    try:
        shape, dtype, device = u.shape, u.dtype, _device()
        if (len(shape) == 3 and shape[1] >= 1 and shape[2] >= 1 and w.shape == shape and w.dtype == dtype and u.is_contiguous() and w.is_contiguous()
                and u.get_device() == w.get_device() == device
                and (v is None or (v.shape == shape and v.dtype == dtype and v.is_contiguous() and v.get_device() == device))
                and (lengths is None or (lengths.dtype == torch.int32 and lengths.shape == shape[:1] and lengths.is_contiguous() and lengths.get_device() == device))):
            return shape, dtype, _CODE[dtype], _GATES[gate]
    except (AttributeError, TypeError, KeyError):
        pass
    _contiguous("u", u, _IO, 3)
    shape, dtype = u.shape, u.dtype
    _contiguous("w", w, (dtype,), 3, shape)
    if v is not None:
        _contiguous("v", v, (dtype,), 3, shape)
    if lengths is not None:
        _contiguous("lengths", lengths, (torch.int32,), 1, shape[:1])
    if gate not in _GATES:
        raise ValueError("gate is \"sigmoid\" or \"log\"")
    if shape[2] < 1 or shape[1] < 1:
        raise ValueError("u must have one channel and one sample at least")
    return shape, dtype, _CODE[dtype], _GATES[gate]


def gated_scan(u, w, v=None, state=None, lengths=None, gate: str = "sigmoid", keep: bool = False):
    """fftconv_gated_scan: (y, last), or (y, last, kept) with keep=True, of h[t] = a[t] h[t-1] + x[t] along the samples, y = v . h.
    u, w, v: (b, c, n) fp32, fp16 or bf16. gate "sigmoid": a = sigmoid(w), x = (1 - a) u; "log": a = exp(min(w, 0)), x = u. state (b, c) fp32:
    before the first sample (None: zeros); last (b, c): after the last one. lengths (b,) int32: the samples of each sequence, the rest is not
    used and zero in y. kept is what gated_scan_backward takes."""
    shape, dtype, code, kind = _scanned(u, w, v, lengths, gate)
    b, c, n = shape
    if state is not None:
        _contiguous("state", state, _F32, 2, (b, c))
    y = torch.empty_like(u)
    last = u.new_empty((b, c), dtype=torch.float32)
    kept = u.new_empty((b, c, -(-n // 512)), dtype=torch.float32) if keep else None
    if b:
        lib = _f.load()
        need = _workspace(lib, "gated_scan", b, c, n, code)
        ws = u.new_empty(need, dtype=torch.uint8) if need else None
        rc = _calls(lib).gated_scan(u.data_ptr(), w.data_ptr(), _ptr(v), _ptr(state), _ptr(lengths), y.data_ptr(), last.data_ptr(), _ptr(kept), b, c, n,
                                    kind, code, _ptr(ws), _f._stream_ptr())
        if rc:
            _f._check(rc)
    return (y, last, kept) if keep else (y, last)


def gated_scan_backward(dy, u, w, kept, v=None, dlast=None, lengths=None, gate: str = "sigmoid"):
    """fftconv_gated_scan_backward: (d, dstate); d (3, b, c, n), the gradients of u, w and v one after the other, (2, b, c, n) without v, so that
    du, dw, dv = d, and what takes a projection's parts takes d. dlast (b, c) fp32: the gradient of `last` (None: zeros); dstate (b, c) fp32."""
    shape, dtype, code, kind = _scanned(u, w, v, lengths, gate)
    b, c, n = shape
    _contiguous("dy", dy, (dtype,), 3, shape)
    _contiguous("kept", kept, _F32, 3, (b, c, -(-n // 512)))
    if dlast is not None:
        _contiguous("dlast", dlast, _F32, 2, (b, c))
    d = u.new_empty((2 if v is None else 3, b, c, n))
    dstate = u.new_empty((b, c), dtype=torch.float32)
    if b:
        lib = _f.load()
        need = _workspace(lib, "gated_scan", b, c, n, code)
        ws = u.new_empty(need, dtype=torch.uint8) if need else None
        at, size = d.data_ptr(), dy.numel() * dy.element_size()
        rc = _calls(lib).gated_scan_backward(dy.data_ptr(), u.data_ptr(), w.data_ptr(), _ptr(v), kept.data_ptr(), _ptr(dlast), _ptr(lengths), at,
                                             at + size, None if v is None else at + 2 * size, dstate.data_ptr(), b, c, n, kind, code, _ptr(ws),
                                             _f._stream_ptr())
        if rc:
            _f._check(rc)
    return d, dstate


def gated_step(u, w, state, v=None, gate: str = "sigmoid", out=None):
    """fftconv_gated_step: y of one sample for every channel, u, w, v and state of one shape ((b, c), say). The state after it replaces `state`, or
    goes to `out`, where both have to be kept; `out` overlaps none of the others."""
    if out is None:
        out = state
    try:
        shape, dtype, device = u.shape, u.dtype, _device()
        code, kind = _CODE[dtype], _GATES[gate]
        good = (w.shape == state.shape == out.shape == shape and w.dtype == dtype and state.dtype == out.dtype == torch.float32 and u.is_contiguous()
                and w.is_contiguous() and state.is_contiguous() and out.is_contiguous()
                and u.get_device() == w.get_device() == state.get_device() == out.get_device() == device
                and (v is None or (v.shape == shape and v.dtype == dtype and v.is_contiguous() and v.get_device() == device)))
    except (AttributeError, TypeError, KeyError):
        good = False
    if not good:                                  # one after the other, for what is wrong
        _contiguous("u", u, _IO)
        shape, dtype = u.shape, u.dtype
        _contiguous("w", w, (dtype,), None, shape)
        if v is not None:
            _contiguous("v", v, (dtype,), None, shape)
        _contiguous("state", state, _F32, None, shape)
        _contiguous("out", out, _F32, None, shape)
        raise ValueError("gate is \"sigmoid\" or \"log\"")
    y = torch.empty_like(u)
    t = y.numel()
    if t:
        rc = _calls(_f.load()).gated_step(u.data_ptr(), w.data_ptr(), _ptr(v), state.data_ptr(), out.data_ptr(), y.data_ptr(), t, kind, code,
                                          _f._stream_ptr())
        if rc:
            _f._check(rc)
    return y


def quantize_blocks(x, layout: str = "tokens", parts: int = 1):
    """fftconv_quantize_blocks: rows x (..., k) in e4m3 with a scale for each 128 of them (Blocks8), what linear_f8 takes. layout "channels":
    fftconv_quantize_blocks_channels, of x (b, k, n), or (parts, b, k / parts, n) with parts > 1; q is (b, n, k) either way."""
    if layout == "tokens" and parts == 1:
        t, k, ldx = _rows("x", x)
        shape, dtype, device = x.shape, x.dtype, x.device
        q = torch.empty_like(x, dtype=_F8, memory_format=torch.contiguous_format) if ldx == k else _empty(shape, dtype=_F8, device=device)
        scale = x.new_empty((-(-k // 128), *shape[:-1]), dtype=torch.float32)
        if t:
            rc = _calls(_f.load()).quantize_blocks(x.data_ptr(), ldx, q.data_ptr(), scale.data_ptr(), t, k, _CODE[dtype], _f._stream_ptr())
            if rc:
                _f._check(rc)
        return Blocks8(q, scale)
    parts = int(parts)
    if layout != "channels" or parts < 1:
        raise ValueError("layout is \"tokens\" or \"channels\", parts 1 for tokens")
    _contiguous("x", x, _IO, 4 if parts > 1 else 3)
    if parts > 1 and x.shape[0] != parts:
        raise ValueError("x must be (parts, b, channels, n)")
    b, c, n = x.shape[-3:]
    k = parts * c
    if k < 1 or n < 1:
        raise ValueError("x must have one channel and one sample at least")
    q = _empty((b, n, k), dtype=_F8, device=x.device)
    scale = _empty((-(-k // 128), b, n), dtype=torch.float32, device=x.device)
    if b:
        rc = _calls(_f.load()).quantize_blocks_channels(x.data_ptr(), q.data_ptr(), scale.data_ptr(), b, n, k, parts, _CODE[x.dtype], _f._stream_ptr())
        if rc:
            _f._check(rc)
    return Blocks8(q, scale)


def quantize_tiles(w, transposed: bool = False):
    """fftconv_quantize_tiles: a weight (o, k) in e4m3 with a scale for each 128 x 128 (Tiles8), once for every call until it changes. With transposed=True
    a pair, the second one of w^T (k, o), the same values: what the gradient of the projection's input is multiplied with."""
    o, k, ldw = _rows("w", w)
    if w.dim() != 2 or o < 1:
        raise ValueError("w must be (o, k), one output at least")
    to, tk, device = -(-o // 128), -(-k // 128), w.device
    q, scale = _empty((o, k), dtype=_F8, device=device), _empty((to, tk), dtype=torch.float32, device=device)
    qt = scale_t = None
    if transposed:
        qt, scale_t = _empty((k, o), dtype=_F8, device=device), _empty((tk, to), dtype=torch.float32, device=device)
    rc = _calls(_f.load()).quantize_tiles(w.data_ptr(), ldw, q.data_ptr(), scale.data_ptr(), _ptr(qt), _ptr(scale_t), o, k, _CODE[w.dtype], _f._stream_ptr())
    if rc:
        _f._check(rc)
    return (Tiles8(q, scale), Tiles8(qt, scale_t)) if transposed else Tiles8(q, scale)


def _f8_operands(xq, xs, wq, ws):
    """(o, k) of a projection's operands. (All checks together, 1.4 us where one after the other they take 2.6 of the 9.8 of a call on one row; what does not
    pass is gone through once more for what is wrong with it.)"""
    try:
        (o, k), device = wq.shape, _device()
        blocks = -(-k // 128)
        if (xq.dtype == wq.dtype == _F8 and xs.dtype == ws.dtype == torch.float32 and xq.is_contiguous() and wq.is_contiguous() and xs.is_contiguous()
                and ws.is_contiguous() and xq.get_device() == wq.get_device() == xs.get_device() == ws.get_device() == device and xq.dim() in (2, 3)
                and xq.shape[-1] == k >= 1 and o >= 1 and xs.shape == (blocks, *xq.shape[:-1]) and ws.shape == (-(-o // 128), blocks)):
            return o, k
    except (AttributeError, TypeError, ValueError):
        pass
    _contiguous("rows", xq, (_F8,))
    if xq.dim() not in (2, 3):
        raise ValueError("rows must be (b, n, k) or (t, k)")
    _contiguous("weight", wq, (_F8,), 2)
    o, k = wq.shape
    if xq.shape[-1] != k or k < 1 or o < 1:
        raise ValueError("rows and weight differ in length, or have none")
    blocks = -(-k // 128)
    _contiguous("the rows' scale", xs, _F32, None, (blocks, *xq.shape[:-1]))
    _contiguous("the weight's scale", ws, _F32, None, (-(-o // 128), blocks))
    return o, k


def linear_f8(rows, weight, bias=None, dtype=torch.bfloat16, layout: str = "tokens", parts: int = 1):
    """fftconv_linear_f8: rows (b, n, k) (or (t, k): one sequence), Blocks8 or a pair (q, scale), and weight (o, k), Tiles8 or a pair; bias (o,) fp32.
    layout "tokens": y (b, n, o). "channels": y (b, o, n), or (parts, b, o / parts, n) with parts > 1."""
    (xq, xs), (wq, ws) = rows, weight
    o, k = _f8_operands(xq, xs, wq, ws)
    if bias is not None:
        _contiguous("bias", bias, _F32, 1, (o,))
    if dtype not in _CODE:
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
    y = xq.new_empty(shape, dtype=dtype)
    if y.numel() == 0:
        return y
    p, code, lib = 0 if layout == "tokens" else parts, _CODE[dtype], _f.load()
    need = _workspace(lib, "linear_f8", b, n, k, o, p, code)
    work = xq.new_empty(need, dtype=torch.uint8) if need else None
    rc = _calls(lib).linear_f8(xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), _ptr(bias), y.data_ptr(), b, n, k, o, p, code, _ptr(work),
                               _f._stream_ptr())
    if rc:
        _f._check(rc)
    return y


def _tensors(name, ts):
    """Addresses, counts and type codes of contiguous tensors on the current device, as arrays. (The checks of all of them together: 12 tensors take 2 us
    instead of the 4.6 of a call for each.)"""
    try:
        good = all(map(torch.Tensor.is_contiguous, ts)) and (not ts or set(map(torch.Tensor.get_device, ts)) == {_device()})
        types = array.array("i", [_CODE[t.dtype] for t in ts])
    except (TypeError, KeyError):
        good = False
    if not good:
        for t in ts:
            _contiguous(name, t, _IO)
    return array.array("Q", map(torch.Tensor.data_ptr, ts)), array.array("q", map(torch.Tensor.numel, ts)), types


def _clip(grads, max_norm, out, norm, eps, write):
    grads = list(grads)
    at, counts, types = _tensors("a gradient", grads)
    to, types_to, result = None, None, norm
    if write:
        to, types_to = at, types
        if out is not None:
            out = list(out)
            if len(out) != len(grads):
                raise ValueError("out must have a tensor for each gradient")
            to, _, types_to = _tensors("a tensor of out", out)
            if [o.shape for o in out] != [t.shape for t in grads] or any(b and a != b for a, b in zip(types, types_to)):
                for t, o in zip(grads, out):
                    _contiguous("a tensor of out", o, (t.dtype, torch.float32), None, t.shape)
        if norm is not None:
            _contiguous("norm", norm, _F32)
            if norm.numel() != 1:
                raise ValueError("norm must be one number")
            if not grads:
                return norm
    lib, work, n = _f.load(), None, len(grads)
    address = lambda a: a.buffer_info()[0] if a else None  # noqa: E731
    if norm is None:
        device = grads[0].device if grads else torch.device("cuda", _device())
        result = _empty((), dtype=torch.float32, device=device)
        work = _empty(lib.fftconv_workspace_bytes_clip_grads(address(counts), n), dtype=torch.uint8, device=device)
    rc = lib.fftconv_clip_grads(address(at), address(to), address(counts), address(types), address(types_to), n, max_norm, eps, _ptr(norm),
                                None if norm is not None else result.data_ptr(), _ptr(work), _f._stream_ptr())
    if rc:
        _f._check(rc)
    return result


def grad_norm(grads):
    """fftconv_clip_grads without clipping: the 2-norm over all of the tensors together, () fp32 on the device. grads: any number of contiguous
    tensors of any sizes, each fp32, fp16 or bf16; squares are added in 64 bits."""
    return _clip(grads, 0.0, None, None, 0.0, False)


def clip_grads(grads, max_norm: float, out=None, norm=None, eps: float = 1e-6):
    """fftconv_clip_grads: every gradient times min(1, max_norm / (norm + eps)), in place, or into `out`, a tensor for each of the same shape and type or
    in fp32. norm: what grad_norm gave, or the norm over other devices' gradients too, one fp32 on the device outside of
    what is written; None: that of grads. Returns the norm."""
    return _clip(grads, float(max_norm), out, norm, float(eps), True)

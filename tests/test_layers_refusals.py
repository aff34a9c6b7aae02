"""What the operators around the convolutions refuse, before any device is touched: through the C ABI, and in the binding."""
import ctypes

import pytest
import torch

from paper_2311_05908_amd import fftconv, layers

F32, F16, BF16 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED = 0, -1, -2
A = 4096          # an address that is aligned and never read


def call(name, *a):
    lib = fftconv.load()
    rc = getattr(lib, name)(*a)
    if rc != OK:
        assert name in lib.fftconv_last_error().decode()
    return rc


def norm(x=A, ldx=64, r=None, ldr=0, w=A, y=A, h=None, rstd=None, scale=None, t=2, d=64, eps=1e-6, dtype=BF16):
    return call("fftconv_rms_norm", x, ldx, r, ldr, w, y, h, rstd, scale, t, d, eps, dtype, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(y=None), EINVAL), (dict(ldx=63), EINVAL), (dict(r=A, ldr=63), EINVAL), (dict(t=-1), EINVAL),
    (dict(t=1 << 31), EINVAL), (dict(d=0), EINVAL), (dict(d=-5), EINVAL), (dict(dtype=3), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(x=A + 1), EINVAL), (dict(x=A + 2, dtype=F32), EINVAL), (dict(w=A + 2), EINVAL),
    (dict(y=A + 1), EINVAL), (dict(h=A + 1), EINVAL), (dict(rstd=A + 2), EINVAL), (dict(scale=A + 1), EINVAL),
    (dict(d=16385, ldx=20000), EUNSUPPORTED), (dict(t=0, x=None, y=None, w=None), OK),
])
def test_norm(kw, rc):
    assert norm(**kw) == rc


def back(dy=A, lddy=64, h=A, dh=None, w=A, rstd=A, dx=A, dw=A, t=2000, d=64, dtype=BF16, ws=A):
    return call("fftconv_rms_norm_backward", dy, lddy, h, dh, w, rstd, dx, dw, t, d, dtype, ws, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dy=None), EINVAL), (dict(h=None), EINVAL), (dict(w=None), EINVAL), (dict(rstd=None), EINVAL), (dict(dx=None), EINVAL), (dict(dw=None), EINVAL),
    (dict(ws=None), EINVAL), (dict(lddy=10), EINVAL), (dict(dtype=-1), EINVAL), (dict(t=-1), EINVAL), (dict(dh=A + 1), EINVAL), (dict(ws=A + 1), EINVAL),
    (dict(d=16385, lddy=20000), EUNSUPPORTED),
])
def test_norm_backward(kw, rc):
    assert back(**kw) == rc


def test_quantize_rows():
    def q(x=A, ld=64, o=A, s=A, t=2, d=64, dtype=F16):
        return call("fftconv_quantize_rows", x, ld, o, s, t, d, dtype, None)
    for kw in (dict(x=None), dict(o=None), dict(s=None), dict(ld=3), dict(dtype=9), dict(s=A + 1), dict(d=0)):
        assert q(**kw) == EINVAL, kw
    assert q(d=1 << 20, ld=1 << 20) == EUNSUPPORTED and q(t=0) == OK


def linear(x=A, xs=A, w=A, ws=A, bias=None, y=A, b=2, n=3, k=64, o=12, parts=0, dtype=BF16, work=A):
    return call("fftconv_linear_i8", x, xs, w, ws, bias, y, b, n, k, o, parts, dtype, work, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(x=None), EINVAL), (dict(xs=None), EINVAL), (dict(w=None), EINVAL), (dict(ws=None), EINVAL), (dict(y=None), EINVAL), (dict(parts=5), EINVAL),
    (dict(parts=-1), EINVAL), (dict(b=-1), EINVAL), (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(o=0), EINVAL), (dict(b=1 << 20, n=1 << 12), EINVAL),
    (dict(o=1 << 31), EINVAL), (dict(dtype=4), EINVAL), (dict(xs=A + 2), EINVAL), (dict(bias=A + 1), EINVAL), (dict(y=A + 1), EINVAL),
    (dict(k=131072), EUNSUPPORTED), (dict(b=0, x=None, y=None), OK),
])
def test_linear(kw, rc):
    assert linear(**kw) == rc


def test_checkpoints():
    def pack(x=A, q=A, s=A, b=2, c=3, n=100, tokens=0, dtype=F32):
        return call("fftconv_act_pack", x, q, s, b, c, n, tokens, dtype, None)

    def unpack(q=A, s=A, gq=None, gs=None, g=None, x=A, b=2, c=3, n=100, dtype=F32):
        return call("fftconv_act_unpack", q, s, gq, gs, g, x, b, c, n, dtype, None)

    huge = dict(b=1 << 30, c=1 << 30, n=1 << 30)
    for kw in (dict(x=None), dict(q=None), dict(s=None), dict(b=-1), dict(c=0), dict(n=0), dict(dtype=3), dict(x=A + 2), dict(s=A + 2), huge):
        assert pack(**kw) == EINVAL, kw
    for kw in (dict(x=None), dict(q=None), dict(s=None), dict(gq=A), dict(gs=A), dict(gq=A, gs=A, g=A), dict(dtype=3), dict(g=A + 1), huge):
        assert unpack(**kw) == EINVAL, kw
    assert pack(b=0) == OK and unpack(b=0) == OK


def weight(dy=A, q=A, s=A, dw=A, b=2, n=100, o=5, c=6, tokens=1, dtype=BF16, out=F32, work=A):
    return call("fftconv_linear_grad_weight", dy, q, s, dw, b, n, o, c, tokens, dtype, out, work, None)


@pytest.mark.parametrize("kw", [
    dict(dy=None), dict(q=None), dict(s=None), dict(dw=None), dict(work=None), dict(b=-1), dict(n=0), dict(o=0), dict(c=0), dict(dtype=3), dict(out=F16),
    dict(dtype=F32, out=BF16), dict(o=1 << 31), dict(b=1 << 24, n=1 << 20), dict(dy=A + 1), dict(s=A + 2), dict(dw=A + 2), dict(work=A + 2),
])
def test_weight_gradient(kw):
    assert weight(**kw) == EINVAL


def test_weight_gradient_of_sizes_beyond_its_kernels():
    assert weight(n=(1 << 22) + 1) == weight(o=1 << 23) == weight(c=1 << 23) == EUNSUPPORTED


def test_workspaces_of_what_is_refused_are_empty():
    lib = fftconv.load()
    assert lib.fftconv_workspace_bytes_rms_norm_backward(-1, 64, BF16) == 0
    assert lib.fftconv_workspace_bytes_rms_norm_backward(100000, 64, 7) == 0
    assert lib.fftconv_workspace_bytes_linear_i8(1, 1, 0, 5, 0, BF16) == 0
    assert lib.fftconv_workspace_bytes_linear_grad_weight(1, 1, 0, 5, 0, BF16) == 0
    assert lib.fftconv_workspace_bytes_rms_norm_backward(100000, 64, BF16) % (64 * 4) == 0


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, w = torch.zeros(2, 4, 8), torch.ones(8)
    q, s = torch.zeros(2, 4, 8, dtype=torch.int8), torch.zeros(2, 4, 1)
    for f in (lambda: layers.rms_norm(x, w), lambda: layers.rms_norm_i8(x, w), lambda: layers.rms_norm_backward(x, x, w, s[..., 0]), lambda: layers.quantize_rows(x),
              lambda: layers.linear_i8((q, s[..., 0]), (q[0], s[0, :, 0])), lambda: layers.act_pack(x), lambda: layers.act_unpack((q, s)),
              lambda: layers.linear_grad_weight(x, (q, s))):
        with pytest.raises(ValueError):
            f()


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_would_misread():
    d = "cuda"
    x, w = torch.zeros(2, 4, 8, device=d), torch.ones(8, device=d)
    q, s = torch.zeros(2, 4, 8, dtype=torch.int8, device=d), torch.zeros(2, 4, device=d)
    wq, ws = torch.zeros(6, 8, dtype=torch.int8, device=d), torch.zeros(6, device=d)
    cs = torch.zeros(2, 4, 1, device=d)
    y, h, rstd = layers.rms_norm(x, w)
    bad = [
        lambda: layers.rms_norm(x.double(), w), lambda: layers.rms_norm(x, w[:7]), lambda: layers.rms_norm(x, w.half()), lambda: layers.rms_norm(x, w.cpu()),
        lambda: layers.rms_norm(x.transpose(1, 2), torch.ones(4, device=d)), lambda: layers.rms_norm(x, w, residual=x.half()),
        lambda: layers.rms_norm(x, w, residual=x[:1]), lambda: layers.rms_norm(torch.zeros(2, 3, 8, device=d)[:, ::2].expand(2, 2, 8)[:, :1].expand(2, 3, 8), w),
        lambda: layers.rms_norm(torch.tensor(1.0, device=d), w), lambda: layers.rms_norm(x[..., :0], w[:0]),
        lambda: layers.rms_norm_backward(x, h.half(), w, rstd), lambda: layers.rms_norm_backward(x, h, w, rstd[:1]),
        lambda: layers.rms_norm_backward(x, h, w, rstd, dh=h[..., :4]),
        lambda: layers.linear_i8((q.float(), s), (wq, ws)), lambda: layers.linear_i8((q, s[:1]), (wq, ws)), lambda: layers.linear_i8((q, s), (wq[:, :7], ws)),
        lambda: layers.linear_i8((q, s), (wq, ws[:5])), lambda: layers.linear_i8((q, s), (wq, ws), bias=ws.half()),
        lambda: layers.linear_i8((q, s), (wq, ws), layout="rows"), lambda: layers.linear_i8((q, s), (wq, ws), parts=2),
        lambda: layers.linear_i8((q, s), (wq, ws), layout="channels", parts=4), lambda: layers.linear_i8((q, s), (wq, ws), dtype=torch.int8),
        lambda: layers.linear_i8((q[0, 0], s[0, 0]), (wq, ws)),
        lambda: layers.act_pack(x[0]), lambda: layers.act_pack(x.transpose(1, 2)), lambda: layers.act_pack(x, layout="rows"), lambda: layers.act_pack(x.int()),
        lambda: layers.act_unpack((q, s)), lambda: layers.act_unpack((q, cs[:1])), lambda: layers.act_unpack((q, cs), dtype=torch.int32),
        lambda: layers.act_unpack((q, cs), gate=x), lambda: layers.act_unpack((q, cs), gate=(q[:1], cs[:1])),
        lambda: layers.linear_grad_weight(x[:1], (q, cs)), lambda: layers.linear_grad_weight(x.transpose(1, 2), (q, cs)),
        lambda: layers.linear_grad_weight(torch.zeros(2, 8, 5, device=d), (q, cs), dtype=torch.float16),
        lambda: layers.linear_grad_weight(torch.zeros(2, 8, 5, device=d), (q, cs), layout="channels"),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail("call %d was taken" % i)
    with pytest.raises(ValueError):
        layers.rms_norm(torch.zeros(1, 8, device=d).expand(4, 8), w)          # rows on top of each other
    with pytest.raises(fftconv.FFTConvError):
        layers.rms_norm(torch.zeros(1, 16385, device=d), torch.ones(16385, device=d))


def test_the_extension_passes_a_norms_arguments():
    """Thirteen integers with a double among them, through the call that the norm is made with; refused in other numbers or kinds."""
    from paper_2311_05908_amd import build

    if build.build_fastcall() is None:
        pytest.skip("no Python headers")
    from paper_2311_05908_amd import _fastcall

    seen = []
    i64 = [ctypes.c_int64]
    f = ctypes.CFUNCTYPE(ctypes.c_int, *i64 * 11, ctypes.c_double, *i64 * 2)(lambda *a: seen.append(a) or -3)
    address = ctypes.cast(f, ctypes.c_void_p).value
    given = [0x7f1234567890, -1, None, 0, 5, 6, None, 8, 9, 1 << 40, 11, 2, 0x7f0000000010]
    assert _fastcall.call_norm(address, 1e-6, *given) == -3
    want = [x or 0 for x in given]
    assert seen == [(*want[:11], 1e-6, *want[11:])]
    for bad in ([1e-6, *given[:-1]], [1e-6, *given, 0], ["x", *given], [None, *given], [1e-6, *given[:-1], 1.5], [1e-6, *given[:-1], 1 << 64]):
        with pytest.raises((TypeError, OverflowError)):
            _fastcall.call_norm(address, *bad)
    with pytest.raises(ValueError):
        _fastcall.call_norm(0, 1e-6, *given)
    for n in (13, 14):
        seen.clear()
        g = ctypes.CFUNCTYPE(ctypes.c_int, *i64 * n)(lambda *a: seen.append(a) or n)
        assert _fastcall.call(ctypes.cast(g, ctypes.c_void_p).value, *range(1, n + 1)) == n and seen == [tuple(range(1, n + 1))]

"""Sizes that the operators around the convolutions refuse because a count would leave 32 bits, before any device is touched; and their binding with an
extension from before them."""
import types

import pytest

from paper_2311_05908_amd import fftconv, layers
from test_layers_refusals import BF16, EINVAL, EUNSUPPORTED, F32, linear, weight

TOP = 1 << 31


@pytest.mark.parametrize("kw", [dict(b=TOP // 512 - 1, n=513), dict(b=TOP - 511, n=1), dict(b=1, n=TOP - 1), dict(o=TOP - 511), dict(o=TOP - 1)])
def test_projections_whose_last_tile_would_end_beyond_32_bits(kw):
    """b n up to 2^31 - 512, and so with o: from there on the row behind a tile of 256, and a store of eight, is a number of 32 bits."""
    assert linear(**kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(b=1 << 20, n=(1 << 11) - 1, o=TOP - 512), dict(b=1, n=TOP - 512, o=1 << 12), dict(b=1 << 11, n=1 << 12, o=(1 << 19) + 1, dtype=F32)])
def test_projections_of_more_tiles_than_32_bits_count(kw):
    assert linear(**{"dtype": BF16, **kw}) == EUNSUPPORTED


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b", [0, 2])
def test_weight_gradients_of_more_tiles_than_a_launch_has_threads_for(b, dtype):
    for o, c in ((1 << 22, (1 << 14) + 1), ((1 << 18) + 1, 1 << 18), (1 << 22, 1 << 22)):
        assert weight(b=b, o=o, c=c, dtype=dtype) == EUNSUPPORTED


def test_an_extension_from_before_these_operators_is_not_called(monkeypatch):
    """Its call() refuses their 13 and 14 arguments: every entry point is then called through ctypes."""
    def old(address, *a):
        raise TypeError("call: no entry point takes %d arguments" % len(a))

    monkeypatch.setattr(fftconv, "_extension", lambda: types.SimpleNamespace(call=old))
    assert fftconv._fastcall.__wrapped__() is None
    monkeypatch.setattr(fftconv, "_fastcall", fftconv._fastcall.__wrapped__)
    monkeypatch.setattr(fftconv, "_entry", fftconv._entry.__wrapped__)
    lib = fftconv.load()
    calls = layers._calls.__wrapped__(lib)
    assert calls.linear_grad_weight is lib.fftconv_linear_grad_weight and calls.act_unpack is lib.fftconv_act_unpack
    assert calls.linear_i8(None, None, None, None, None, None, 0, 1, 1, 1, 0, BF16, None, None) == 0
    assert calls.rms_norm(1e-6, None, 8, None, 0, None, None, None, None, None, 0, 8, BF16, None) == 0
    assert calls.rms_norm(-1.0, None, 8, None, 0, None, None, None, None, None, 0, 8, BF16, None) == EINVAL

"""Sizes that the operators around the convolutions refuse because a count would leave 32 bits, before any device is touched."""
import pytest

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

"""The operators around the convolutions on the GPU where a size, a place or a value is at the end of what a call takes. Tolerances as in
test_layers_gpu.py."""
import pytest
import torch

from paper_2311_05908_amd import layers
from test_layers_gpu import DT, RUN, gen, normal, runs8, weight_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(1, 65, 1, 40), (2, 70, 1, 7), (3, 134, 1, 130), (1, 66, 2, 33), (2, 129, 3, 20), (1, 193, 2, 128), (1, 71, 1, 5), (2, 80, 3, 16)])
def test_weight_gradient_of_few_channels(b, n, o, c, layout, dtype):
    """Less than 8 channels of dy and a few samples behind a half run: the last piece of a sample reaches over several of those."""
    g = gen(b + n + o + c)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n))
    weight_check(dy, q, s, layout, "f32")
    assert torch.equal(layers.linear_grad_weight(dy, (q, s), layout=layout, dtype=DT[dtype]), layers.linear_grad_weight(dy, (q, s), layout=layout).to(DT[dtype]))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(2, 1200, 72, 140), (2, 1201, 72, 140), (1, 128, 16, 8), (3, 656, 1032, 1030), (3, 655, 1032, 1030), (1, 16, 8, 2), (1, 3, 2, 1)])
def test_weight_gradient_where_a_scale_is_zero(b, n, o, c, layout, dtype):
    """q is not zero there: a run whose scale is zero stands for zeros all the same, be it the first of a channel, one between others, the last, several,
    or all."""
    g = gen(21)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n) * torch.exp(3 * normal(g, b, c, 1)))
    s[0, 0::6, 0] = 0
    s[-1, 1::6, -1] = 0
    s[:, 2::6, s.shape[-1] // 2] = 0
    s[:, 3::6, 1::2] = 0
    s[:, 4::12] = 0
    got = weight_check(dy, q, s, layout, "f32")
    assert c <= 4 or bool((got[:, 4::12] == 0).all())
    assert torch.equal(got, layers.linear_grad_weight(dy, (q * (s != 0).repeat_interleave(RUN, -1)[..., :n], s), layout=layout))

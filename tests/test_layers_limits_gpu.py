"""The operators around the convolutions on the GPU where a size, a place or a value is at the end of what a call takes. Tolerances as in
test_layers_gpu.py."""
import pytest
import torch

from paper_2311_05908_amd import layers
from test_layers_gpu import DT, gen, normal, runs8, weight_check

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

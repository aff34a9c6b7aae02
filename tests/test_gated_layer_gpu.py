"""examples/gated_layer.py: the operators around the convolution and the convolution together, against the layer in 64 bits without any 8-bit rounding.

The bounds: eight bits of values whose largest is m times their root mean square (m below 6 here, 4 to 5 in rows and runs this long) are off by
m / 127 / sqrt(12), under 1.4 % of it; products of three such, sums of many, and bf16 between them (0.4 % for a convolution) stay under
sqrt(6) 1.4 % + 1 %, 5 % of the result's root mean square."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("gated_layer", os.path.join(ROOT, "examples", "gated_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(layer, x, r, norm, w_in, k):
    """y (b, d, n) and h in 64 bits."""
    h = x + r
    z = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6) * norm
    u, w, v = (z @ w_in.T).transpose(1, 2).chunk(3, 1)
    fft = layer.plan.fft_size
    conv = torch.fft.irfft(torch.fft.rfft(u * w, fft) * torch.fft.rfft(k, fft), fft)[..., : layer.n]
    return v * conv, h


def off(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("batch,samples,channels", [(3, 1000, 96), (2, 2048, 256)])
def test_layer(batch, samples, channels):
    layer = example().GatedLayer(channels, samples, seed=samples)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dh = (torch.randn(batch, samples, channels, generator=g, device="cuda").to(layer.dtype) for _ in range(3))
    dy = torch.randn(batch, channels, samples, generator=g, device="cuda").to(layer.dtype)
    leaves = [t.double().requires_grad_(True) for t in (x, r, layer.norm, layer.w_in, layer.k)]
    y, h = plain(layer, *leaves)
    ((y * dy.double()).sum() + (h * dh.double()).sum()).backward()
    got, hg, kept = layer.train_forward(x, r)
    assert off(got, y.detach()) < 0.05 and off(hg, h.detach()) < 0.004
    dx, dnorm, dw_in, dk = layer.backward(kept, dy, dh=dh)
    for name, a, b in (("dx", dx, leaves[0].grad), ("dnorm", dnorm, leaves[2].grad), ("dw_in", dw_in, leaves[3].grad), ("dk", dk, leaves[4].grad)):
        print(name, off(a, b))
        assert torch.isfinite(a.float()).all() and off(a, b) < 0.05, name
    out, h8 = layer.forward(x, r)
    assert torch.equal(h8, hg) and off(out, y.detach().transpose(1, 2) @ layer.w_out.double().T) < 0.05

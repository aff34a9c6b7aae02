"""On the GPU: results that overlap what else a call of the recurrent layer's operators reads or writes are refused and leave everything as it was; tensors side by
side in one buffer are taken and give the bits of tensors apart."""
import pytest
import torch

from paper_2311_05908_amd import fftconv, layers

pytestmark = pytest.mark.gpu


def side_by_side(ts):
    """Copies of tensors, one where the other ends (behind a first value, so that none is aligned to more than its elements)."""
    size = ts[0].element_size()
    store = torch.empty(size + sum(t.numel() * t.element_size() for t in ts), dtype=torch.uint8, device="cuda")
    at, views = size, []
    for t in ts:
        n = t.numel() * t.element_size()
        views.append(store[at:at + n].view(t.dtype).view(t.shape).copy_(t))
        at += n
    return views


def test_step():
    g = torch.Generator(device="cuda").manual_seed(1)
    u, w, v, state = (torch.randn(7, 1001, generator=g, device="cuda") for _ in range(4))
    kept = [t.clone() for t in (u, w, v, state)]
    out = torch.empty_like(state)
    y = layers.gated_step(u, w, state, v=v, out=out)
    for t in (u, w, v):
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, state, v=v, out=t)
    both = torch.zeros(8, 1001, device="cuda")
    both[:7] = state
    for a, b in ((both[:7], both[1:]), (both[1:], both[:7])):
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, a, v=v, out=b)
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, state, v=a, out=b)
    assert all(torch.equal(a, b) for a, b in zip((u, w, v, state), kept)) and not both[7].any()
    a, b, c, d, e = side_by_side([u, out, w, state, v])
    assert torch.equal(layers.gated_step(a, c, d, v=e, out=b), y) and torch.equal(b, out)
    assert all(torch.equal(x, k) for x, k in zip((a, c, e, d), kept))
    assert torch.equal(layers.gated_step(a, c, d, v=e), y) and torch.equal(d, out)          # in place

"""Projections from e4m3 with long rows on the GPU, within bounds in which a part of k that is left out shows (that it does is tested beside this, on the CPU)."""
import pytest
import torch

from linear_f8_bounds import F8, LONG, block_sums, operands, value_and_bound
from paper_2311_05908_amd import layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,k,o", LONG)
def test_long_rows(t, k, o):
    rows, weight = operands(t, k, o, "cuda", seed=k + o)
    sums = block_sums(rows, weight)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        y, bound = value_and_bound(sums, dtype)
        for layout in ("tokens", "channels"):
            got = layers.linear_f8(rows, weight, dtype=dtype, layout=layout)
            assert got.dtype == dtype
            over = ((got if layout == "tokens" else got.t()).double() - y).abs() - bound
            assert float(over.max()) <= 0, "%s, %s: %g over at %d of %d places" % (dtype, layout, float(over.max()), int((over > 0).sum()), over.numel())


@pytest.mark.parametrize("t", [1, 40, 300, 2048])
def test_what_products_of_eight_neighbours_lose(t):
    """One product of 2^16 beside one of 1.875^2 2^a: what is below 2^3 is lost to 16-bit results, toward zero, where both are among the same eight of k, and
    nothing elsewhere or to fp32 results. (The large one is taken away again in the next block.)"""
    o, k = 128, 256
    for a in range(-4, 12):
        for sign in (1, -1):
            xv, wv = 1.875 * 2.0 ** max(-4, min(7, a)), sign * 1.875 * 2.0 ** (a - max(-4, min(7, a)))
            for place in (1, 7, 8, 64):
                x, w = torch.zeros(t, k, device="cuda"), torch.zeros(o, k, device="cuda")
                x[:, 0], x[:, 128], w[:, 0], w[:, 128] = 256, 256, 256, -256
                x[:, place], w[:, place] = xv, wv
                rows, weight = (x.to(F8), torch.ones(2, t, device="cuda")), (w.to(F8), torch.ones(1, 2, device="cuda"))
                exact = xv * wv
                kept = (abs(exact) // 8 * 8) * sign
                y = layers.linear_f8(rows, weight, dtype=torch.bfloat16)
                if place < 8:
                    assert bool((y == torch.tensor(kept).bfloat16().cuda()).all()), (a, sign, place, float(y[0, 0]), kept)
                else:                             # (as fp32 has it beside 2^16: steps of 2^-7)
                    assert bool(((y.float() - exact).abs() <= 2.0 ** -7 + 2.0 ** -8 * abs(exact)).all()), (a, sign, place, float(y[0, 0]), exact)
                z = layers.linear_f8(rows, weight, dtype=torch.float32)
                assert bool(((z - exact).abs() <= 2.0 ** -7).all())

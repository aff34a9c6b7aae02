"""The bounds that projections from e4m3 with long rows are held to see what a kernel might get wrong: planted here in results made on the CPU."""
import pytest
import torch

from linear_f8_bounds import LONG, block_sums, operands, value_and_bound


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,k,o", LONG)
def test_a_part_left_out_shows(t, k, o, dtype):
    """Some tokens and outputs of each: the value rounded is within its bound; zeros, and what is left without any one of the shortest ranges (four blocks, or 1/256
    of k), or with one of them added twice, are outside at some place."""
    rows, weight = operands(min(t, 4), k, min(o, 12), "cpu", seed=k + o)
    sums = block_sums(rows, weight)
    y, bound = value_and_bound(sums, dtype)
    off = lambda z: bool(((z.to(dtype).double() - y).abs() > bound).any())  # noqa: E731
    assert not off(y) and off(torch.zeros_like(y))
    blocks = sums.shape[-1]
    per = max(4, -(-blocks // 256))
    for first in range(0, blocks, per):
        part = sums[0, :, :, first:first + per].sum(-1)
        assert off(y - part) and off(y + part), (first, per)

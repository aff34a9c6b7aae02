"""The operators of a recurrent layer, in the release build and in the one with full barriers and waits (see test_sync_check_gpu.py): bit for bit."""
import pytest
import torch

from paper_2311_05908_amd import build as hip_build
from paper_2311_05908_amd import fftconv

pytestmark = pytest.mark.gpu


def test_operators_of_a_recurrent_layer_agree_bit_for_bit(monkeypatch):
    """Projections from e4m3 on both tiles, in both layouts, whole and with edges, in ranges, of few tokens, through registers; quantisers; the scan."""
    from paper_2311_05908_amd import layers

    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)

    # (rows, samples, k, outputs, parts)
    shapes = [(4, 4096, 768, 2304, 3), (2, 2048, 768, 2304, 3), (1, 8190, 528, 4000, 1), (1, 100, 4096, 2048, 2), (1, 5, 1000, 100, 1), (1, 777, 333, 555, 1), (3, 999, 400, 600, 2),
              (1, 1, 700, 16400, 1), (1, 9, 1100, 8200, 1), (1, 20, 300, 8200, 1), (1, 50, 300, 8200, 2), (1, 50, 300, 16400, 2), (1, 40, 8192, 300, 1), (1, 40, 256, 33000, 1)]
    cases = [(normal(b, n, k), normal(o, k), parts) for b, n, k, o, parts in shapes]
    u, w, v, dy = (normal(3, 40, 5000) for _ in range(4))
    grads = [normal(1000), normal(300, 77)]
    out = []
    for lib in (fftconv.load(), fftconv.load(hip_build.LIB_SYNC_CHECK)):
        monkeypatch.setattr(fftconv, "load", lambda path=None: lib)
        got = []
        for x, weight, parts in cases:
            rows, (tiles, tiles_t) = layers.quantize_blocks(x), layers.quantize_tiles(weight, transposed=True)
            y = layers.linear_f8(rows, tiles, layout="channels", parts=parts)
            back = layers.quantize_blocks(y, layout="channels", parts=parts)
            got += [rows.q.float(), rows.scale, y, back.q.float(), back.scale, tiles_t.q.float(), layers.linear_f8(rows, tiles), layers.linear_f8(back, tiles_t)]
            got += [layers.linear_f8(rows, tiles, dtype=torch.float32), layers.linear_f8(rows, tiles, dtype=torch.float32, layout="channels", parts=parts)]
        y, last, kept = layers.gated_scan(u, w, v=v, keep=True)
        d, dstate = layers.gated_scan_backward(dy, u, w, kept, v=v)
        to = [torch.empty_like(t) for t in grads]
        got += [y, last, kept, d, dstate, layers.clip_grads(grads, 1.0, out=to), *to]
        out.append(got)
        torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*out)):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b), i

"""The operators around the convolutions, in the release build and in the one with full barriers and waits (see test_sync_check_gpu.py): bit for bit."""
import torch
import pytest

from paper_2311_05908_amd import build as hip_build
from paper_2311_05908_amd import fftconv

pytestmark = pytest.mark.gpu


def test_operators_around_the_convolutions_agree_bit_for_bit(monkeypatch):
    """Norm, 8-bit projections on their tiles and in ranges, checkpoints, and the weight's gradient on both of its kernels."""
    from paper_2311_05908_amd import layers

    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)

    x, r, gate, w = normal(4, 4096, 768), normal(4, 4096, 768), normal(4, 768, 4096), normal(1536, 768)
    norm = torch.ones(768, device="cuda")
    wide = normal(1, 100, 4096), normal(2048, 4096)
    out = []
    for lib in (fftconv.load(), fftconv.load(hip_build.LIB_SYNC_CHECK)):
        monkeypatch.setattr(fftconv, "load", lambda path=None: lib)
        y, h, rstd = layers.rms_norm(x, norm, residual=r)
        rows, _, _ = layers.rms_norm_i8(x, norm, residual=r)
        w8 = layers.quantize_rows(w)
        u = layers.linear_i8(rows, w8, layout="channels", parts=2)
        p = layers.act_pack(y, layout="tokens")
        odd = layers.act_pack(y[:, :4001].contiguous(), layout="tokens")
        out.append((y, h, rstd, *rows, *w8, u, layers.linear_i8(rows, w8, dtype=torch.float32), layers.linear_i8(*(layers.quantize_rows(t) for t in wide)),
                    *p, layers.act_unpack(p, gate=gate), *layers.rms_norm_backward(r, h, norm, rstd), layers.linear_grad_weight(x, p),
                    layers.linear_grad_weight(gate, p, layout="channels"), layers.linear_grad_weight(x[:, :4001].contiguous(), odd)))
        torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*out)):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b), i

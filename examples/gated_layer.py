#!/usr/bin/env python3
"""A gated long-convolution layer from the library's operators: serving in 8 bits, and a training step that keeps its activations in 8 bits.

    h = x + r;  z = norm(h);  u, w, v = z W^T;  y = v . ((u . w) * k);  out = y W_out^T

    python examples/gated_layer.py [--batch 8 --samples 2048 --channels 768]

forward() is the layer as it answers: the norm leaves its rows in 8 bits, the projection multiplies them with an 8-bit weight and writes u, w and
v channel by channel, as the convolution takes them. train_forward() is the same up to the convolution, and keeps z, u, w and v in 8 bits (half of
their 16); backward() returns the gradients of x, the norm's weight, W and k, recomputing what was not kept. Gradients pass the 8-bit roundings as
if they were not there.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2311_05908_amd import fftconv, layers  # noqa: E402


class GatedLayer:
    def __init__(self, channels: int, samples: int, seed: int = 0, dtype=torch.bfloat16, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        fft = max(256, 1 << (2 * samples - 1).bit_length())
        self.d, self.n, self.dtype = channels, samples, dtype
        self.plan = fftconv.Plan(samples, fft, channels, dtype)
        self.norm = torch.ones(channels, device=device)
        self.w_in = torch.randn(3 * channels, channels, generator=g, device=device) / channels ** 0.5
        self.w_out = torch.randn(channels, channels, generator=g, device=device) / channels ** 0.5
        decay = torch.exp(-torch.linspace(4 / samples, 40 / samples, channels, device=device)[:, None] * torch.arange(samples, device=device))
        self.k = torch.randn(channels, samples, generator=g, device=device) * decay / 8
        self.weights_changed()

    def weights_changed(self):
        """What is made once of the weights, for every call until they change."""
        self.w_in8, self.w_out8 = layers.quantize_rows(self.w_in), layers.quantize_rows(self.w_out)
        self.kf, self.kf_adjoint = self.plan.filter_fft(self.k), self.plan.filter_fft_adjoint(self.k)

    def forward(self, x, r):
        """x, r (b, n, d) -> out (b, n, d), h (b, n, d), the residual stream for the next layer."""
        rows, h, _ = layers.rms_norm_i8(x, self.norm, residual=r)
        u, w, v = layers.linear_i8(rows, self.w_in8, dtype=self.dtype, layout="channels", parts=3)
        y = self.plan.forward_gated(u, w, v, self.kf)
        return layers.linear_i8(layers.quantize_rows(y.transpose(1, 2).contiguous()), self.w_out8, dtype=self.dtype), h

    def train_forward(self, x, r):
        """The layer up to the convolution's result y (b, d, n), and what backward() takes."""
        z, h, rstd = layers.rms_norm(x, self.norm, residual=r)
        u, w, v = layers.linear_i8(layers.quantize_rows(z), self.w_in8, dtype=self.dtype, layout="channels", parts=3)
        y = self.plan.forward_gated(u, w, v, self.kf)
        kept = {"h": h, "rstd": rstd, "z": layers.act_pack(z, layout="tokens")}
        kept.update(u=layers.act_pack(u), w=layers.act_pack(w), v=layers.act_pack(v))
        return y, h, kept

    def backward(self, kept, dy, dh=None):
        """dy (b, d, n), the gradient of y; dh, that of h. Returns dx, dnorm, dw_in, dk."""
        b, dt = dy.shape[0], self.dtype
        uw = layers.act_unpack(kept["u"], dtype=dt, gate=kept["w"])
        dyv = layers.act_unpack(kept["v"], dtype=dt, gate=dy)
        duw = self.plan.backward_input(dyv, self.kf_adjoint)
        dk = self.plan.backward_filter(uw, dyv, self.k.shape[1])
        duwv = torch.cat([layers.act_unpack(kept["w"], dtype=dt, gate=duw), layers.act_unpack(kept["u"], dtype=dt, gate=duw),
                          dy * self.plan.forward(uw, self.kf)], 1)
        dw_in = layers.linear_grad_weight(duwv, kept["z"], layout="channels")
        dz = (duwv.transpose(1, 2).reshape(-1, 3 * self.d) @ self.w_in.to(dt)).reshape(b, self.n, self.d)
        dx, dnorm = layers.rms_norm_backward(dz, kept["h"], self.norm, kept["rstd"], dh=dh)
        return dx, dnorm, dw_in, dk


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--samples", type=int, default=2048)
    ap.add_argument("--channels", type=int, default=768)
    a = ap.parse_args()
    layer = GatedLayer(a.channels, a.samples)
    x, r, dy = (torch.randn(a.batch, a.samples, a.channels, device="cuda").to(layer.dtype) for _ in range(3))
    dy = dy.transpose(1, 2).contiguous()

    def timed(f):
        for _ in range(3):
            f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t) / 10 * 1e3

    def step():
        _, _, kept = layer.train_forward(x, r)
        return layer.backward(kept, dy)

    bits16 = 4 * x.numel() * 2
    _, _, kept = layer.train_forward(x, r)
    bits8 = sum(t.numel() * t.element_size() for name in "zuwv" for t in kept[name])
    print("%d x %d x %d: forward in 8 bits %.3f ms, training step %.3f ms, kept activations %.1f MB instead of %.1f" % (
        a.batch, a.samples, a.channels, timed(lambda: layer.forward(x, r)), timed(step), bits8 / 1e6, bits16 / 1e6))


if __name__ == "__main__":
    main()

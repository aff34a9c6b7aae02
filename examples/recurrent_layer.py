#!/usr/bin/env python3
"""A gated layer with a recurrence in the place of the long convolution, from the library's operators: prompts and single tokens with a state between
them, and a training step with projections in 8-bit floating point.

    h = x + r;  z = norm(h);  u, w, v = z W^T + b;  s[t] = a[t] s[t-1] + (1 - a[t]) u[t], a = sigmoid(w);  y = v . s;  out = y W_out^T

    python examples/recurrent_layer.py [--batch 8 --samples 2048 --channels 768]

forward() answers a batch of prompts, of lengths of their own, and returns the state after each; step() goes on by one token. Both use the weights in e4m3,
a scale for each 128 x 128, as train_forward() and backward() do, which multiply with their transposes too. Gradients pass the 8-bit roundings as if
they were not there; update() clips them by their norm and steps.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2311_05908_amd import layers  # noqa: E402


class RecurrentLayer:
    def __init__(self, channels: int, seed: int = 0, dtype=torch.bfloat16, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.d, self.dtype = channels, dtype
        self.norm = torch.ones(channels, device=device)
        self.w_in = torch.randn(3 * channels, channels, generator=g, device=device) / channels ** 0.5
        self.w_out = torch.randn(channels, channels, generator=g, device=device) / channels ** 0.5
        # memories from a few samples to a thousand
        self.b_in = torch.zeros(3 * channels, device=device)
        self.b_in[channels:2 * channels] = torch.linspace(1, 7, channels, device=device)
        self.weights_changed()

    def weights_changed(self):
        """What is made once of the weights, for every call until they change."""
        self.in8, self.in8_t = layers.quantize_tiles(self.w_in, transposed=True)
        self.out8, self.out8_t = layers.quantize_tiles(self.w_out, transposed=True)

    def forward(self, x, r, state=None, lengths=None):
        """x, r (b, n, d) -> out (b, n, d), h (b, n, d), the residual stream for the next layer, and the state (b, d) after each sequence."""
        z, h, _ = layers.rms_norm(x, self.norm, residual=r)
        u, w, v = layers.linear_f8(layers.quantize_blocks(z), self.in8, bias=self.b_in, dtype=self.dtype, layout="channels", parts=3)
        y, state = layers.gated_scan(u, w, v=v, state=state, lengths=lengths)
        return layers.linear_f8(layers.quantize_blocks(y, layout="channels"), self.out8, dtype=self.dtype), h, state

    def step(self, x, r, state):
        """x, r (b, d), one token for each sequence -> out, h (b, d); the state goes on in place."""
        z, h, _ = layers.rms_norm(x, self.norm, residual=r)
        rows = layers.quantize_blocks(z.unsqueeze(1))
        u, w, v = layers.linear_f8(rows, self.in8, bias=self.b_in, dtype=self.dtype, layout="channels", parts=3).squeeze(-1)
        y = layers.gated_step(u, w, state, v=v)
        return layers.linear_f8(layers.quantize_blocks(y), self.out8, dtype=self.dtype), h

    def train_forward(self, x, r):
        """out, h and what backward() takes."""
        z, h, rstd = layers.rms_norm(x, self.norm, residual=r)
        u, w, v = layers.linear_f8(layers.quantize_blocks(z), self.in8, bias=self.b_in, dtype=self.dtype, layout="channels", parts=3)
        y, _, states = layers.gated_scan(u, w, v=v, keep=True)
        out = layers.linear_f8(layers.quantize_blocks(y, layout="channels"), self.out8, dtype=self.dtype)
        kept = {"h": h, "rstd": rstd, "z": layers.act_pack(z, layout="tokens"), "y": layers.act_pack(y), "states": states, "uwv": (u, w, v)}
        return out, h, kept

    def backward(self, kept, dout, dh=None):
        """dout (b, n, d), the gradient of out; dh, that of h. Returns dx and the gradients of norm, w_in, b_in and w_out."""
        u, w, v = kept["uwv"]
        dy = layers.linear_f8(layers.quantize_blocks(dout), self.out8_t, dtype=self.dtype, layout="channels")
        d, _ = layers.gated_scan_backward(dy, u, w, kept["states"], v=v)
        dz = layers.linear_f8(layers.quantize_blocks(d, layout="channels", parts=3), self.in8_t, dtype=self.dtype)
        dx, dnorm = layers.rms_norm_backward(dz, kept["h"], self.norm, kept["rstd"], dh=dh)
        dw_in = torch.cat([layers.linear_grad_weight(t, kept["z"], layout="channels") for t in d])
        db_in = d.float().sum((1, 3)).flatten()
        return dx, [dnorm, dw_in, db_in, layers.linear_grad_weight(dout, kept["y"])]

    def update(self, grads, rate: float, limit: float = 1.0):
        """A step against the gradients, clipped by their norm, which is returned."""
        norm = layers.clip_grads(grads, limit)
        for p, g in zip((self.norm, self.w_in, self.b_in, self.w_out), grads):
            p.sub_(g, alpha=rate)
        self.weights_changed()
        return norm


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--samples", type=int, default=2048)
    ap.add_argument("--channels", type=int, default=768)
    a = ap.parse_args()
    layer = RecurrentLayer(a.channels)
    x, r, dout = (torch.randn(a.batch, a.samples, a.channels, device="cuda").to(layer.dtype) for _ in range(3))

    def timed(f):
        for _ in range(3):
            f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - t) / 10 * 1e3

    def train():
        _, _, kept = layer.train_forward(x, r)
        layer.update(layer.backward(kept, dout)[1], 0.0)

    _, _, state = layer.forward(x, r)
    token = x[:, 0].contiguous(), r[:, 0].contiguous()
    print("%d x %d x %d: forward %.3f ms, a token more %.3f ms, training step %.3f ms" % (
        a.batch, a.samples, a.channels, timed(lambda: layer.forward(x, r)), timed(lambda: layer.step(*token, state)), timed(train)))


if __name__ == "__main__":
    main()

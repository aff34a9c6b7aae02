"""The work that the layers around a long convolution have the 8-bit and norm operators do, as a list of cases with their inputs,
one pass, its unavoidable work and its result from the definition in 64 bits.

The operators (t tokens = b sequences of n samples, d channels in, o channels out):
  norm         h = x + r; y = h / sqrt(mean(h^2) + eps) * w                       the residual's addition and the norm, one pass forward
  norm train   the same, and its backward pass: dx (for x and r alike), dw        h comes in rounded to the I/O type, as it was kept
  norm linear  the norm with y in 8 bits, a scale for each token, and the product with an 8-bit weight, a scale for each output channel
  linear       the product alone, its result token by token (b, n, o) or channel by channel (parts, b, o / parts, n), the layout that the
               convolutions take (parts = 3: u, w and v of a gated convolution)
  checkpoint   x (b, c, n) packed into 8 bits with a scale for every 128 samples of a channel, and read back for the backward pass, alone or
               as the product with a second one (u . w, which the gradient of a gated convolution's filter takes)
  weight       the gradient of a projection's weight, dw[o, c] = sum over b, n of dy[b, n, o] x[b, c, n], x from 8 bits
"""
from __future__ import annotations

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
RUN = 128            # samples that share a scale in a checkpoint
LEAST = 2.0 ** -100  # rows and runs whose largest magnitude is below this are zeros with a scale of zero


def _norm(op, dtype, t, d, o=0, b=1, layout="tokens", parts=1):
    return {"op": op, "dtype": dtype, "b": b, "n": t // b, "d": d, "o": o, "layout": layout, "parts": parts}


def listed():
    return [
        # generating text, one sequence: the norm before a layer on a single token, where the time to launch counts
        dict(_norm("norm", "bf16", 1, 768), name="norm bf16 1 x 768"),
        # a prompt of a length that nobody chose, with channels that fill no vector, half precision
        dict(_norm("norm", "f16", 5 * 1999, 1001, b=5), name="norm f16 5 x 1999 x 1001"),
        # training a 768-channel layer on a batch of 4K sequences
        dict(_norm("norm train", "bf16", 64 * 4096, 768, b=64), name="norm train bf16 64 x 4096 x 768"),
        # a reference run in fp32, wide rows, an odd number of tokens
        dict(_norm("norm train", "f32", 3 * 1365, 4096, b=3), name="norm train f32 3 x 1365 x 4096"),
        # generating text, one sequence, a wide layer: norm and projection of a single token, bound by the weight's bytes
        dict(_norm("norm linear", "bf16", 1, 4096, 4096), name="norm linear bf16 1 x 4096 -> 4096"),
        # one prompt into a gated convolution: norm and projection to u, w and v
        dict(_norm("norm linear", "bf16", 4096, 768, 2304, b=2, layout="channels", parts=3), name="norm linear bf16 2 x 2048 x 768 -> 3 x 768"),
        # the same projection of the headline batch of 4K sequences
        dict(_norm("linear", "bf16", 64 * 4096, 768, 2304, b=64, layout="channels", parts=3), name="linear bf16 64 x 4096 x 768 -> 3 x 768"),
        # a wide layer's expansion over a long prompt, bound by the matrix cores
        dict(_norm("linear", "f16", 8192, 4096, 16384), name="linear f16 8192 x 4096 -> 16384"),
        # a small fp32 model's activations, rows that end inside a run
        dict(_norm("checkpoint", "f32", 2 * 1000, 16, b=2), parts=1, name="checkpoint f32 2 x 16 x 1000"),
        # two operands of a gated layer of the headline shape
        dict(_norm("checkpoint", "bf16", 64 * 4096, 768, b=64), parts=2, name="checkpoint bf16 64 x 768 x 4096 gated"),
        # one odd prompt, fp16 gradients as the convolution's backward pass leaves them
        dict(_norm("weight", "f16", 2047, 768, 768, layout="channels"), name="weight f16 2047 x 768 -> 768"),
        # the gradient of the projection of the headline batch
        dict(_norm("weight", "bf16", 64 * 4096, 768, 2304, b=64), name="weight bf16 64 x 4096 x 768 -> 2304"),
    ]


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def draw(rng):
    """One more case of the ranges above: 1 to 2^18 tokens, 16 to 8192 channels, odd ones among both, every operator, layout and type."""
    while True:
        op = rng.choice(["norm", "norm train", "norm linear", "linear", "linear", "checkpoint", "weight", "weight"])
        # (activations of an fp32 model are not taken to 8 bits on the way forward: the steps are a thousand times what fp32 resolves)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32" if op != "norm linear" else "bf16"])
        n = int(2 ** rng.uniform(0, 15))
        b = max(1, int(2 ** rng.uniform(-3, 6)))
        if op == "weight":
            n += 63
        d = int(2 ** rng.uniform(6, 13)) if op != "checkpoint" else int(2 ** rng.uniform(4, 10))
        o = int(2 ** rng.uniform(6, 14))
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
            o = max(64, o // 64 * 64)
        layout, parts = rng.choice([("tokens", 1), ("channels", 1), ("channels", 3)])
        if op == "weight" and parts == 3:
            layout, parts = "tokens", 1
        if op == "checkpoint":
            layout, parts = "channels", rng.choice([1, 2])
        if op in ("norm", "norm train"):
            layout, parts = "tokens", 1
        if op in ("norm", "norm train", "checkpoint"):
            o = 0
        elif parts == 3:
            o = max(1, o // 3) * 3
        if 3072 in (d, o, n, b * n):
            continue
        c = _norm(op, dtype, b * n, d, o, b=b, layout=layout, parts=parts)
        w = work(c)
        # in bytes no more than the largest listed case of its kind, in operations than the largest one
        if w["bytes"] <= 1.4e9 and w["flops"] <= 1.09e12 and b * n * max(d, o) <= 64 * 4096 * 2304:
            return c


def _rows8(x):
    """Rows in 8 bits with a scale each: q = round(x / s) to even, s = max |x| / 127. (Both quotients of tensors: torch makes a product with the
    reciprocal of a quotient by a number, which is not the same in the last bit.)"""
    x = x.float()
    top = x.abs().amax(-1)
    s = torch.where(top < LEAST, torch.zeros_like(top), top / torch.full_like(top, 127))
    q = torch.round(x / torch.where(s == 0, torch.ones_like(s), s)[..., None])
    return torch.where((s == 0)[..., None], torch.zeros_like(q), q), s


def _runs8(x):
    """Runs of 128 samples of each channel in 8 bits: x (b, c, n) -> q (b, c, n), s (b, c, runs)."""
    b, c, n = x.shape
    runs = -(-n // RUN)
    q, s = _rows8(torch.nn.functional.pad(x.float(), (0, runs * RUN - n)).reshape(b, c, runs, RUN))
    return q.reshape(b, c, runs * RUN)[..., :n], s


def _from_runs(q, s):
    return q.float() * s.repeat_interleave(RUN, -1)[..., : q.shape[-1]]


def prepare(case, seed):
    """Activations, weights and gradients as the layers have them: one channel in a hundred is twenty times as large as the others
    (as it is in trained models), norm weights are near one, projections keep the size of what passes them; 8-bit weights are quantised
    once, for every call after."""
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    b, n, d, o, dtype = c["b"], c["n"], c["d"], c["o"], DTYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    big = 1.0 + 19.0 * (torch.rand(d, generator=g, device=dev) < 0.01)
    s = {"case": c}
    if c["op"].startswith("norm"):
        s["x"], s["r"] = (normal(b, n, d) * big).to(dtype), (normal(b, n, d) * big).to(dtype)
        s["weight"] = 1 + 0.1 * normal(d)
    if c["op"] == "norm train":
        s["dy"], s["dh"] = normal(b, n, d).to(dtype), normal(b, n, d).to(dtype)
    if c["op"] in ("norm linear", "linear"):
        q, s["ws"] = _rows8(normal(o, d) / d ** 0.5)
        s["wq"], s["bias"] = q.to(torch.int8), 0.1 * normal(o)
    if c["op"] == "linear":
        q, s["xs"] = _rows8(normal(b, n, d) * big)
        s["xq"] = q.to(torch.int8)
    if c["op"] == "checkpoint":
        s["x"] = (normal(b, d, n) * big[:, None]).to(dtype)
        if c["parts"] == 2:
            s["gate"] = normal(b, d, n).to(dtype)
    if c["op"] == "weight":
        s["dy"] = normal(*((b, n, o) if c["layout"] == "tokens" else (b, o, n))).to(dtype)
        q, s["cs"] = _runs8(normal(b, d, n) * big[:, None])
        s["cq"] = q.to(torch.int8)
    return s


def run(state):
    s = state
    c = s["case"]
    op, dtype = c["op"], DTYPES[c["dtype"]]
    return _run_own(s, c, op, dtype) if own else _run_plain(s, c, op, dtype)


def _run_own(s, c, op, dtype):
    from paper_2311_05908_amd import layers

    if op == "norm":
        y, h, _ = layers.rms_norm(s["x"], s["weight"], residual=s["r"], eps=EPS)
        return {"y": y, "h": h}
    if op == "norm train":
        y, h, rstd = layers.rms_norm(s["x"], s["weight"], residual=s["r"], eps=EPS)
        dx, dw = layers.rms_norm_backward(s["dy"], h, s["weight"], rstd, dh=s["dh"])
        return {"y": y, "h": h, "dx": dx, "dw": dw}
    if op == "norm linear":
        rows, h, _ = layers.rms_norm_i8(s["x"], s["weight"], residual=s["r"], eps=EPS)
        return {"h": h, "y": layers.linear_i8(rows, (s["wq"], s["ws"]), bias=s["bias"], dtype=dtype, layout=c["layout"], parts=c["parts"])}
    if op == "linear":
        return {"y": layers.linear_i8((s["xq"], s["xs"]), (s["wq"], s["ws"]), bias=s["bias"], dtype=dtype, layout=c["layout"], parts=c["parts"])}
    if op == "checkpoint":
        p = layers.act_pack(s["x"])
        gate = layers.act_pack(s["gate"]) if c["parts"] == 2 else None
        return {"x": layers.act_unpack(p, dtype=dtype, gate=gate), "scale": p[1]}
    return {"dw": layers.linear_grad_weight(s["dy"], (s["cq"], s["cs"]), layout=c["layout"], dtype=dtype)}


def _laid_out(y, c):
    """(b, n, o) as the case wants it."""
    if c["layout"] == "tokens":
        return y
    b, n, o = y.shape
    y = y.reshape(b, n, c["parts"], o // c["parts"]).permute(2, 0, 3, 1).contiguous()
    return y[0] if c["parts"] == 1 else y


def _run_plain(s, c, op, dtype):
    if op.startswith("norm"):
        h = s["x"].float() + s["r"].float()
        rstd = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
        y, kept = h * rstd * s["weight"], h.to(dtype)
        if op == "norm":
            return {"y": y.to(dtype), "h": kept}
        if op == "norm train":
            hat, g = kept.float() * rstd, s["dy"].float() * s["weight"]
            dx = rstd * (g - hat * (g * hat).mean(-1, keepdim=True)) + s["dh"].float()
            dw = (s["dy"].float() * hat).sum((0, 1))
            return {"y": y.to(dtype), "h": kept, "dx": dx.to(dtype), "dw": dw}
        q, xs = _rows8(y)
    elif op == "linear":
        q, xs = s["xq"].float(), s["xs"]
    if op in ("norm linear", "linear"):
        y = torch.matmul(q, s["wq"].float().t()) * xs[..., None] * s["ws"] + s["bias"]
        y = _laid_out(y.to(dtype), c)
        return {"h": kept, "y": y} if op == "norm linear" else {"y": y}
    if op == "checkpoint":
        q, sc = _runs8(s["x"])
        x = _from_runs(q, sc)
        if c["parts"] == 2:
            x = x * _from_runs(*_runs8(s["gate"]))
        return {"x": x.to(dtype), "scale": sc}
    x = _from_runs(s["cq"], s["cs"]).permute(0, 2, 1).reshape(-1, c["d"])
    dy = s["dy"].float()
    dy = (dy if c["layout"] == "tokens" else dy.permute(0, 2, 1)).reshape(-1, c["o"])
    return {"dw": torch.matmul(dy.t(), x).to(dtype)}


def exact(case, seed):
    """The definitions in 64 bits, on the inputs as prepare() makes them."""
    s, op = prepare(case, seed), case["op"]
    f64 = torch.float64
    if op.startswith("norm"):
        x = s["x"].to(f64) + s["r"].to(f64)
        r = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS)
        y = x * r * s["weight"].to(f64)
        if op == "norm":
            return {"y": y, "h": x}
        if op == "norm train":
            # with h as it is kept, rounded, and z = h r: dx = dh + sum over j of dy_j w_j d(h_j r) / dh
            z, dy = x.to(DTYPES[case["dtype"]]).to(f64) * r, s["dy"].to(f64)
            v = dy * s["weight"].to(f64)
            dx = s["dh"].to(f64) + r * v - r * z * ((v * z).sum(-1, keepdim=True) / case["d"])
            return {"y": y, "h": x, "dx": dx, "dw": torch.einsum("bnd,bnd->d", dy, z)}
    if op in ("norm linear", "linear"):
        if op == "linear":
            v = s["xq"].to(f64) * s["xs"].to(f64)[..., None]
        else:
            step = y.abs().max(-1, keepdim=True).values / 127
            v = torch.round(y / step) * step
        w = s["wq"].to(f64) * s["ws"].to(f64)[:, None]
        y = (v.reshape(-1, case["d"]) @ w.T).reshape(case["b"], case["n"], -1) + s["bias"].to(f64)
        if case["layout"] == "channels":
            y = torch.stack([z.transpose(1, 2) for z in y.chunk(case["parts"], -1)])
            y = y if case["parts"] > 1 else y[0]
        return {"h": x, "y": y} if op == "norm linear" else {"y": y}
    if op == "checkpoint":
        steps, values = [], []
        for t in [s["x"]] + ([s["gate"]] if case["parts"] == 2 else []):
            cut = t.to(f64).split(RUN, -1)
            step = [z.abs().max(-1, keepdim=True).values / 127 for z in cut]
            values.append(torch.cat([torch.round(z / e) * e for z, e in zip(cut, step)], -1))
            steps.append(torch.cat(step, -1))
        return {"x": values[0] * values[1] if len(values) == 2 else values[0], "scale": steps[0]}
    x = s["cq"].to(f64)
    for j in range(s["cs"].shape[-1]):
        x[..., j * RUN:(j + 1) * RUN] *= s["cs"][..., j:j + 1].to(f64)
    dw = torch.zeros(case["o"], case["d"], dtype=f64, device=x.device)
    for b in range(case["b"]):
        dy = s["dy"][b].to(f64)
        dw += (dy.T if case["layout"] == "tokens" else dy) @ x[b].T
    return {"dw": dw}


def work(case):
    """Each input read once and each output written once. Products count two operations for each pair of factors, the rest what the
    formulas hold for each value."""
    t, d, o, size = case["b"] * case["n"], case["d"], case["o"], _size(case)
    runs = case["b"] * d * -(-case["n"] // RUN)
    if case["op"] == "norm":                                    # x, r in; y, h out
        return {"bytes": 4 * t * d * size + 4 * d, "flops": 5 * t * d}
    if case["op"] == "norm train":                              # x, r, dy, dh in; y, h, dx out (h comes from the pass itself)
        return {"bytes": 7 * t * d * size + 8 * d, "flops": 16 * t * d}
    if case["op"] == "norm linear":                             # x, r and the weight in; h, y out
        return {"bytes": 3 * t * d * size + 4 * d + o * d + 8 * o + t * o * size, "flops": 2 * t * d * o + 7 * t * d}
    if case["op"] == "linear":
        return {"bytes": t * d + 4 * t + o * d + 8 * o + t * o * size, "flops": 2 * t * d * o}
    if case["op"] == "checkpoint":                              # x (and the gate) in; 8 bits and scales out and in again; x out
        return {"bytes": case["parts"] * (t * d * (size + 2) + 8 * runs) + t * d * size, "flops": case["parts"] * 5 * t * d}
    return {"bytes": t * o * size + t * d + 4 * runs + o * d * size, "flops": 2 * t * d * o}

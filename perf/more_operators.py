"""A gated recurrence in the place of the long convolution, and what trains and serves such a layer, as a list of cases with their inputs, one pass,
its unavoidable work and its result from the definition in 64 bits.

The operators (b sequences of n samples, c or d channels in, o channels out):
  step          one token for every sequence: h' = a h + x, y = v h', with gates from their logits w: a = sigmoid(w), x = (1 - a) u
  scan          the same over n samples from a state, u, w, v and y (b, c, n) as the convolutions have them; gate "log" takes a = exp(w), x = u instead;
                sequences of a padded batch end where `lengths` says (zeros behind it), the state after the last sample comes back
  scan train    the scan and its gradients: du, dw, dv and, from a state, the state's
  linear        rows to 8-bit floating point (e4m3), a scale for each 128 of a row, times a weight in e4m3 with a scale for each 128 x 128; the result
                token by token (b, n, o) or channel by channel (parts, b, o / parts, n), the layout that recurrences and convolutions take
  linear back   the same from rows that lie channel by channel in parts, (parts, b, d / parts, n), as a scan's gradients do: the gradient of a
                projection's input, the weight transposed when it was quantised
  weight        the weight in e4m3, with its transpose for the backward pass
  clip          the 2-norm over the gradients of all of a model's tensors, and these times min(1, limit / (norm + 1e-6)), into the optimizer's buffers
"""
from __future__ import annotations

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn
BLOCK = 128           # values of a row, and rows and columns of a weight, that share a scale
LEAST = 2.0 ** -100   # blocks whose largest magnitude is below this are zeros with a scale of zero
EPS = 1e-6


def _scan_case(op, dtype, b, c, n, gate="sigmoid", gated=True, state=True, ragged=False):
    return {"op": op, "dtype": dtype, "b": b, "c": c, "n": n, "gate": gate, "gated": gated, "state": state, "ragged": ragged}


def _linear_case(op, dtype, b, n, d, o, layout="tokens", parts=1, bias=True):
    return {"op": op, "dtype": dtype, "b": b, "n": n, "d": d, "o": o, "layout": layout, "parts": parts, "bias": bias}


def _clip_case(dtype, layers, d, n, out="f32", limited=True):
    return {"op": "clip", "dtype": dtype, "layers": layers, "d": d, "n": n, "out": out, "limited": limited}


def listed():
    return [
        # generating text, one sequence: a layer's recurrence on a single token, where the time to launch counts
        dict(_scan_case("step", "bf16", 1, 768, 1), name="step bf16 1 x 768"),
        # a batch of prompts of lengths that nobody chose, one of them empty, padded to the longest; decays by their logarithms, no output gate
        dict(_scan_case("scan", "f16", 5, 100, 1999, gate="log", gated=False, ragged=True), name="scan f16 5 x 100 x 1999 ragged"),
        # the headline batch of 4K sequences, answered
        dict(_scan_case("scan", "bf16", 64, 768, 4096, state=False), name="scan bf16 64 x 768 x 4096"),
        # ... and trained on
        dict(_scan_case("scan train", "bf16", 64, 768, 4096, state=False), name="scan train bf16 64 x 768 x 4096"),
        # one long sequence of a small fp32 model, a stretch of a longer one: few rows
        dict(_scan_case("scan train", "f32", 1, 16, 131072), name="scan train f32 1 x 16 x 131072"),
        # generating text, one sequence, a wide layer: bound by the weight's bytes
        dict(_linear_case("linear", "bf16", 1, 1, 4096, 4096), name="linear bf16 1 x 4096 -> 4096"),
        # one prompt into a gated layer: rows of the norm to u, w and v
        dict(_linear_case("linear", "bf16", 2, 2048, 768, 2304, layout="channels", parts=3), name="linear bf16 2 x 2048 x 768 -> 3 x 768"),
        # a wide layer's expansion over a long prompt, bound by the matrix cores
        dict(_linear_case("linear", "f16", 1, 8192, 4096, 16384), name="linear f16 8192 x 4096 -> 16384"),
        # the gradient of the headline batch's projection to u, w and v
        dict(_linear_case("linear back", "bf16", 64, 4096, 2304, 768, parts=3, bias=False), name="linear back bf16 64 x 4096 x 3 x 768 -> 768"),
        # a wide layer's fp32 weight after an optimizer's step
        dict(_linear_case("weight", "f32", 1, 1, 4096, 16384, bias=False), name="weight f32 4096 -> 16384"),
        # a small model: a dozen gradients, most of them small
        dict(_clip_case("f32", 3, 64, 1000), name="clip f32 3 layers of 64 x 1000"),
        # the gradients of twenty-four layers, bf16 weights with fp32 norms and filters, over the limit
        dict(_clip_case("bf16", 24, 2048, 4096), name="clip bf16 24 layers of 2048 x 4096"),
    ]


def _size(dtype):
    return 4 if dtype == "f32" else 2


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15 if case["op"].startswith("linear") else 0)


def draw(rng):
    """One more case of the ranges above: 1 to 2^18 tokens, 16 to 16384 channels, odd ones among both, every operator, layout and type."""
    largest = max(_cost(c) for c in listed() if c["op"] == "scan train")
    while True:
        op = rng.choice(["step", "scan", "scan train", "scan train", "linear", "linear", "linear back", "weight", "clip"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        b = max(1, int(2 ** rng.uniform(-3, 6)))
        n = int(2 ** rng.uniform(0, 17))
        if op in ("step", "scan", "scan train"):
            c = int(2 ** rng.uniform(4, 13))
            case = _scan_case(op, dtype, b, c, 1 if op == "step" else n, gate=rng.choice(["sigmoid", "sigmoid", "log"]), gated=rng.random() < 0.7,
                              state=op == "step" or rng.random() < 0.5, ragged=op != "step" and b > 1 and rng.random() < 0.4)
            sizes = b * c * n
        elif op == "clip":
            d = int(2 ** rng.uniform(4, 11.5))
            case = _clip_case(dtype, rng.randint(1, 32), d, int(2 ** rng.uniform(6, 14)), out=rng.choice(["f32", "same"]), limited=rng.random() < 0.8)
            sizes = case["layers"] * (4 * d * d + d * case["n"])
        else:
            d, o = int(2 ** rng.uniform(5, 13)), int(2 ** rng.uniform(5, 14))
            if rng.random() < 0.6:
                d, o = max(64, d // 64 * 64), max(64, o // 64 * 64)
            layout, parts = rng.choice([("tokens", 1), ("channels", 1), ("channels", 3)])
            if op == "linear back":
                layout = "tokens"
            if op == "weight":
                b, n, layout, parts = 1, 1, "tokens", 1
            if parts == 3:
                d, o = (max(1, d // 3) * 3, o) if op == "linear back" else (d, max(1, o // 3) * 3)
            case = _linear_case(op, dtype, b, n, d, o, layout=layout, parts=parts, bias=op == "linear" and rng.random() < 0.7)
            sizes = max(b * n * max(d, o), d * o)
        # (no more than the largest listed case in bytes, operations and values)
        if _cost(case) <= largest and sizes <= 64 * 4096 * 2304 and work(case)["flops"] <= 1.2e12:
            return case


def _shapes(case):
    """The gradients of a model's layers: norm, projections in and out, filters; (shape, whether it is kept in fp32)."""
    d, n = case["d"], case["n"]
    return [s for _ in range(case["layers"]) for s in (((d,), True), ((3 * d, d), False), ((d, d), False), ((d, n), True))]


def _blocks8(x):
    """Rows in e4m3 with a scale for each 128 of them: x (..., k) -> q (..., k), s (..., blocks). (A quotient of tensors: a number's reciprocal
    is not the same in the last bit.)"""
    k = x.shape[-1]
    blocks = -(-k // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - k)).unflatten(-1, (blocks, BLOCK))
    s = _scale(x.abs().amax(-1))
    q = (x / torch.where(s == 0, torch.ones_like(s), s)[..., None]) * (s != 0)[..., None]
    return q.flatten(-2)[..., :k].to(F8), s


def _scale(top):
    return torch.where(top < LEAST, torch.zeros_like(top), top / torch.full_like(top, 448))


def _tiles8(w):
    """A weight in e4m3 with a scale for each 128 x 128: w (o, k) -> q (o, k), s (tiles of o, tiles of k)."""
    o, k = w.shape
    to, tk = -(-o // BLOCK), -(-k // BLOCK)
    s = _scale(torch.nn.functional.pad(w.float(), (0, tk * BLOCK - k, 0, to * BLOCK - o)).reshape(to, BLOCK, tk, BLOCK).abs().amax((1, 3)))
    by = s.repeat_interleave(BLOCK, 0)[:o].repeat_interleave(BLOCK, 1)[:, :k]
    return ((w.float() / torch.where(by == 0, torch.ones_like(by), by)) * (by != 0)).to(F8), s


def prepare(case, seed):
    """Inputs as the layers have them: gates whose memory is from a few samples to thousands, by the channel; one channel in a hundred twenty times as
    large as the others; weights that keep the size of what passes them, quantised once, for every call after; gradients of tensors that
    differ in size by orders of magnitude, with a limit above or below their norm."""
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    dtype = DTYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    s = {"case": c}
    if c["op"] in ("step", "scan", "scan train"):
        b, d, n = c["b"], c["c"], c["n"]
        shape = (b, d) if c["op"] == "step" else (b, d, n)
        channel = torch.rand(d, generator=g, device=dev)
        channel = channel if c["op"] == "step" else channel[:, None]
        s["u"] = normal(*shape).to(dtype)
        if c["gate"] == "log":
            s["w"] = (-torch.exp(1 - 8 * channel + 0.5 * normal(*shape))).to(dtype)
        else:
            s["w"] = (7 * channel + normal(*shape)).to(dtype)
        s["v"] = normal(*shape).to(dtype) if c["gated"] else None
        s["state"] = normal(b, d) if c["state"] else None
        if c["op"] == "step":
            s["next"] = torch.empty_like(s["state"])
        else:
            s["lengths"] = None
            if c["ragged"]:
                s["lengths"] = torch.randint(0, n + 1, (b,), generator=g, device=dev, dtype=torch.int32)
                s["lengths"][0], s["lengths"][-1] = n, 0
        if c["op"] == "scan train":
            s["dy"] = normal(*shape).to(dtype)
            s["dlast"] = normal(b, d) if c["state"] else None
    elif c["op"] == "clip":
        grads = []
        for shape, kept in _shapes(c):
            size = torch.exp(3 * torch.rand((), generator=g, device=dev) - 4) / shape[-1] ** 0.5
            grads.append((normal(*shape) * size).to(torch.float32 if kept else dtype))
        s["grads"] = grads
        # the optimizer's buffers: one for all tensors whose weights are kept in fp32, one for the rest; tensors begin where the last one ended
        s["kept"] = torch.empty(sum(t.numel() for t, (_, k) in zip(grads, _shapes(c)) if k), device=dev)
        s["rest"] = torch.empty(sum(t.numel() for t, (_, k) in zip(grads, _shapes(c)) if not k), device=dev,
                                dtype=torch.float32 if c["out"] == "f32" else dtype)
        at, s["out"] = {True: 0, False: 0}, []
        for t, (_, k) in zip(grads, _shapes(c)):
            s["out"].append((s["kept"] if k else s["rest"])[at[k]:at[k] + t.numel()].view(t.shape))
            at[k] += t.numel()
        norm = sum(float(t.double().square().sum()) for t in grads) ** 0.5
        s["limit"] = norm * (0.3 if c["limited"] else 3.0)
    else:
        b, n, d, o = c["b"], c["n"], c["d"], c["o"]
        w = normal(o, d) / d ** 0.5
        if c["op"] == "weight":
            s["w"] = w.to(dtype)
            return s
        s["wq"], s["ws"] = _tiles8(w)
        s["bias"] = 0.1 * normal(o) if c["bias"] else None
        big = 1.0 + 19.0 * (torch.rand(d, generator=g, device=dev) < 0.01)
        if c["op"] == "linear":
            s["x"] = (normal(b, n, d) * big).to(dtype)
        else:
            p = c["parts"]
            s["x"] = (normal(p, b, d // p, n) * big.reshape(p, 1, d // p, 1)).to(dtype)
    return s


def run(state):
    s = state
    c = s["case"]
    out = _run_own(s, c, DTYPES[c["dtype"]]) if own else _run_plain(s, c, DTYPES[c["dtype"]])
    return {k: t for k, t in out.items() if t is not None}


def _run_own(s, c, dtype):
    from paper_2311_05908_amd import layers

    op = c["op"]
    if op == "step":
        y = layers.gated_step(s["u"], s["w"], s["state"], v=s["v"], gate=c["gate"], out=s["next"])
        return {"y": y, "state": s["next"]}
    if op == "scan":
        y, last = layers.gated_scan(s["u"], s["w"], v=s["v"], state=s["state"], lengths=s["lengths"], gate=c["gate"])
        return {"y": y, "last": last}
    if op == "scan train":
        y, last, kept = layers.gated_scan(s["u"], s["w"], v=s["v"], state=s["state"], lengths=s["lengths"], gate=c["gate"], keep=True)
        d, dstate = layers.gated_scan_backward(s["dy"], s["u"], s["w"], kept, v=s["v"], dlast=s["dlast"], lengths=s["lengths"], gate=c["gate"])
        return {"y": y, "last": last, "du": d[0], "dw": d[1], "dv": d[2] if c["gated"] else None, "dstate": dstate if c["state"] else None}
    if op == "clip":
        return {"norm": layers.clip_grads(s["grads"], s["limit"], out=s["out"], eps=EPS), "kept": s["kept"], "rest": s["rest"]}
    if op == "weight":
        (q, scale), (qt, _) = layers.quantize_tiles(s["w"], transposed=True)
        return {"q": q, "scale": scale, "qt": qt}
    if op == "linear back":
        rows = layers.quantize_blocks(s["x"] if c["parts"] > 1 else s["x"][0], layout="channels", parts=c["parts"])
    else:
        rows = layers.quantize_blocks(s["x"])
    return {"y": layers.linear_f8(rows, (s["wq"], s["ws"]), bias=s["bias"], dtype=dtype, layout=c["layout"], parts=c["parts"] if op == "linear" else 1)}


def _composed(a, x):
    """h_t = a_t h_{t-1} + x_t along the last axis, h_{-1} = 0: steps of 1, 2, 4, ... samples composed (a step for a sample would be thousands of
    launches)."""
    shift = 1
    while shift < a.shape[-1]:
        x = torch.cat([x[..., :shift], x[..., shift:] + a[..., shift:] * x[..., :-shift]], -1)
        a = torch.cat([a[..., :shift], a[..., shift:] * a[..., :-shift]], -1)
        shift *= 2
    return x


def _gates(s, c):
    """(a, 1 - a or None) in fp32."""
    w = s["w"].float()
    if c["gate"] == "log":
        return torch.exp(w), None
    return 1 / (1 + torch.exp(-w)), 1 / (1 + torch.exp(w))


def _run_plain(s, c, dtype):
    op = c["op"]
    if op == "step":
        a, rest = _gates(s, c)
        h = a * s["state"] + (s["u"].float() if rest is None else rest * s["u"].float())
        return {"y": (h if s["v"] is None else h * s["v"].float()).to(dtype), "state": h}
    if op in ("scan", "scan train"):
        return _plain_scan(s, c, dtype)
    if op == "clip":
        norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
        scale = torch.clamp(s["limit"] / (norm + EPS), max=1.0).float()
        _ = [torch.mul(t.float(), scale, out=o) for t, o in zip(s["grads"], s["out"])]
        return {"norm": norm.float(), "kept": s["kept"], "rest": s["rest"]}
    if op == "weight":
        q, scale = _tiles8(s["w"])
        return {"q": q, "scale": scale, "qt": q.t().contiguous()}
    x = s["x"]
    if op == "linear back":
        x = x.permute(1, 3, 0, 2).flatten(2)
    q, xs = _blocks8(x)
    x = q.float() * xs.repeat_interleave(BLOCK, -1)[..., : c["d"]]
    w = s["wq"].float() * s["ws"].repeat_interleave(BLOCK, 0)[: c["o"]].repeat_interleave(BLOCK, 1)[:, : c["d"]]
    y = torch.matmul(x, w.t())
    return {"y": _laid_out((y if s["bias"] is None else y + s["bias"]).to(dtype), c)}


def _laid_out(y, c):
    """(b, n, o) as the case wants it."""
    if c["layout"] == "tokens":
        return y
    b, n, o = y.shape
    y = y.reshape(b, n, c["parts"], o // c["parts"]).permute(2, 0, 3, 1).contiguous()
    return y[0] if c["parts"] == 1 else y


def _plain_scan(s, c, dtype):
    a, rest = _gates(s, c)
    u = s["u"].float()
    x = u if rest is None else rest * u
    v = torch.ones_like(u) if s["v"] is None else s["v"].float()
    there = None
    if s["lengths"] is not None:          # behind a sequence's end the state stays what it is
        there = torch.arange(c["n"], device=u.device) < s["lengths"][:, None, None]
        a, x, v = torch.where(there, a, 1.0), torch.where(there, x, 0.0), torch.where(there, v, 0.0)
    if s["state"] is not None:
        x = torch.cat([x[..., :1] + a[..., :1] * s["state"][..., None], x[..., 1:]], -1)
    h = _composed(a, x)
    out = {"y": (h * v).to(dtype), "last": h[..., -1].contiguous()}
    if c["op"] == "scan":
        return out
    dy = s["dy"].float()
    g = dy * v
    if s["dlast"] is not None:
        g = torch.cat([g[..., :-1], g[..., -1:] + s["dlast"][..., None]], -1)
    after = torch.cat([a[..., 1:], torch.zeros_like(a[..., :1])], -1)
    dh = _composed(after.flip(-1), g.flip(-1)).flip(-1)
    first = torch.zeros_like(h[..., :1]) if s["state"] is None else s["state"][..., None]
    before = torch.cat([first, h[..., :-1]], -1)
    if rest is None:
        du, dw = dh, dh * before * a
    else:
        du, dw = dh * rest, dh * (before - u) * a * rest
    dv = dy * h
    if there is not None:
        du, dw, dv = (torch.where(there, t, 0.0) for t in (du, dw, dv))
    return {**out, "du": du.to(dtype), "dw": dw.to(dtype), "dv": dv.to(dtype) if c["gated"] else None,
            "dstate": a[..., 0] * dh[..., 0] if c["state"] else None}


def exact(case, seed):
    """The definitions in 64 bits, on the inputs as prepare() makes them."""
    s, op, f64 = prepare(case, seed), case["op"], torch.float64
    if op in ("step", "scan", "scan train"):
        return _exact_scan(s, case)
    if op == "clip":
        total = torch.zeros((), dtype=f64, device="cuda")
        for t in s["grads"]:
            total += torch.linalg.vector_norm(t.to(f64)) ** 2
        norm = total ** 0.5
        scale = min(1.0, s["limit"] / (float(norm) + EPS))
        return {"norm": norm, **{name: torch.cat([t.flatten().to(f64) * scale for t, (_, k) in zip(s["grads"], _shapes(case)) if k is kept])
                                 for name, kept in (("kept", True), ("rest", False))}}
    if op == "weight":
        w = s["w"].to(f64)
        scale = torch.stack([torch.stack([t.abs().max() / 448 for t in r.split(BLOCK, 1)]) for r in w.split(BLOCK, 0)])
        q = torch.cat([torch.cat([_e4m3(t / scale[i, j]) for j, t in enumerate(r.split(BLOCK, 1))], 1) for i, r in enumerate(w.split(BLOCK, 0))], 0)
        return {"q": q, "scale": scale, "qt": q.T}
    d, x = case["d"], s["x"].to(f64)
    if op == "linear back":
        x = torch.cat([p.transpose(1, 2) for p in x], -1)
    for i in range(0, d, BLOCK):
        part = x[..., i:i + BLOCK]
        step = part.abs().max(-1, keepdim=True).values / 448
        x[..., i:i + BLOCK] = _e4m3(part / step) * step
    w = s["wq"].to(f64)
    for i in range(s["ws"].shape[0]):
        for j in range(s["ws"].shape[1]):
            w[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK] *= s["ws"][i, j].to(f64)
    y = (x.reshape(-1, d) @ w.T).reshape(case["b"], case["n"], -1)
    if s["bias"] is not None:
        y += s["bias"].to(f64)
    if case["layout"] == "channels":
        y = torch.stack([z.transpose(1, 2) for z in y.chunk(case["parts"], -1)])
        y = y if case["parts"] > 1 else y[0]
    return {"y": y}


def _e4m3(x):
    """x rounded to the numbers of e4m3: three bits behind the first, steps of 2^-9 below 2^-6, ties to even."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))), min=-6.0) - 3)
    return torch.round(x / step) * step


def _one_by_one(a, x, h0):
    """h_t = a_t h_{t-1} + x_t from h0, sample by sample within stretches that are walked side by side, then stretch by stretch."""
    b, c, n = a.shape
    length = max(1, int(n ** 0.5))
    stretches = -(-n // length)
    pad = stretches * length - n
    a = torch.nn.functional.pad(a, (0, pad), value=1.0).reshape(b, c, stretches, length).movedim(-1, 0).contiguous()
    x = torch.nn.functional.pad(x, (0, pad)).reshape(b, c, stretches, length).movedim(-1, 0).contiguous()
    for t in range(1, length):
        x[t] += a[t] * x[t - 1]
        a[t] *= a[t - 1]
    starts = [h0]
    for j in range(stretches - 1):
        starts.append(x[-1, ..., j] + a[-1, ..., j] * starts[-1])
    x += a * torch.stack(starts, -1)
    return x.movedim(0, -1).reshape(b, c, -1)[..., :n]


def _exact_scan(s, case):
    f64 = torch.float64
    u, w = s["u"].to(f64), s["w"].to(f64)
    v = None if s["v"] is None else s["v"].to(f64)
    a = torch.exp(w) if case["gate"] == "log" else torch.sigmoid(w)
    x = u.clone() if case["gate"] == "log" else torch.sigmoid(-w) * u
    if case["op"] == "step":
        h = a * s["state"].to(f64) + x
        return {"y": h if v is None else h * v, "state": h}
    b, c, n = u.shape
    h0 = torch.zeros(b, c, dtype=f64, device=u.device) if s["state"] is None else s["state"].to(f64)
    ends = [n] * b if s["lengths"] is None else s["lengths"].tolist()
    for i, end in enumerate(ends):
        a[i, :, end:], x[i, :, end:] = 1, 0
    h = _one_by_one(a, x, h0)
    y = h.clone() if v is None else h * v
    for i, end in enumerate(ends):
        y[i, :, end:] = 0
    out = {"y": y, "last": h[..., -1].clone()}
    if case["op"] == "scan":
        return out
    dy = s["dy"].to(f64)
    g = dy.clone() if v is None else dy * v
    dv = dy * h
    dlast = torch.zeros_like(h0) if s["dlast"] is None else s["dlast"].to(f64)
    for i, end in enumerate(ends):
        g[i, :, end:], dv[i, :, end:] = 0, 0
    # p_t = a_t dh_t, what reaches the sample before: p_t = a_t (g_t + p_{t+1})
    p = _one_by_one(a.flip(-1), (a * g).flip(-1), dlast).flip(-1)
    dh = g + torch.cat([p[..., 1:], dlast[..., None]], -1)
    q = dh * (torch.cat([h0[..., None], h[..., :-1]], -1) - (0 if case["gate"] == "log" else u)) * a
    if case["gate"] == "log":
        du, dw = dh, q
    else:
        du, dw = dh * torch.sigmoid(-w), q * torch.sigmoid(-w)
    for i, end in enumerate(ends):
        du[i, :, end:], dw[i, :, end:] = 0, 0
    out.update(du=du, dw=dw, dv=dv if case["gated"] else None, dstate=p[..., 0].clone() if case["state"] else None)
    return {k: t for k, t in out.items() if t is not None}


def work(case):
    """Each input read once and each output written once. Products count two operations for each pair of factors, the rest what the
    formulas hold for each value. (Of a ragged batch the whole is counted: what lies behind an end is written, though not read.)"""
    op, size = case["op"], _size(case["dtype"])
    if op in ("step", "scan", "scan train"):
        rows, gated, state = case["b"] * case["c"], int(case["gated"]), int(case["state"])
        t = rows * case["n"]
        if op == "scan train":            # u, w, v, dy in; y, du, dw, dv out
            return {"bytes": (6 + 2 * gated) * t * size + rows * (4 + 12 * state), "flops": 30 * t}
        return {"bytes": (3 + gated) * t * size + rows * (4 + 4 * state), "flops": 8 * t}
    if op == "clip":
        kept = sum(torch.Size(s).numel() for s, k in _shapes(case) if k)
        rest = sum(torch.Size(s).numel() for s, k in _shapes(case) if not k)
        read = 4 * kept + size * rest
        return {"bytes": read + (4 * (kept + rest) if case["out"] == "f32" else read) + 4, "flops": 3 * (kept + rest)}
    t, d, o = case["b"] * case["n"], case["d"], case["o"]
    tiles = -(-d // BLOCK) * -(-o // BLOCK)
    if op == "weight":
        return {"bytes": d * o * (size + 2) + 4 * tiles, "flops": 2 * d * o}
    return {"bytes": t * d * size + o * d + 4 * tiles + 4 * o * int(case["bias"]) + t * o * size, "flops": 2 * t * d * o}

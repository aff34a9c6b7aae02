"""The operators around the convolutions on the GPU, against their definitions in 64 bits.

Tolerances come from the arithmetic: every result is rounded once to its type (half a unit in the last place, U), everything before that is
fp32 (E = 2^-24 an operation). A sum of n terms in fp32, in whatever order, is within n E of the sum of the terms' magnitudes. fp16
results below its normal range are within half its smallest number, TINY."""
import numpy as np
import pytest
import torch

from paper_2311_05908_amd import layers

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}
E = 2.0 ** -24
RUN = 128


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def within(y, ref, bound, what=""):
    y, ref, bound = y.double(), ref.double(), bound.double() if isinstance(bound, torch.Tensor) else bound
    assert y.shape == ref.shape, (what, y.shape, ref.shape)
    assert torch.isfinite(y).all(), what
    over = (y - ref).abs() - bound
    assert y.numel() == 0 or float(over.max()) <= 0, "%s: %g over the bound at %d of %d places" % (
        what, float(over.max()), int((over > 0).sum()), over.numel())


def in_range(x, dtype="f16"):
    """What an fp16 result can hold: beyond its largest number it is an infinity, taken here as that number on both sides."""
    return x.clamp(-65504, 65504) if (x.dtype == torch.float16 or (x.dtype == torch.float64 and dtype == "f16")) else x


def rows8(x):
    """(q, scale) of rows, the quotients rounded to fp32 once (of 64-bit quotients, whose own rounding cannot change that of fp32 numbers)."""
    x = x.float()
    top = x.abs().amax(-1)
    s = torch.where(top < 2.0 ** -100, torch.zeros_like(top), (top.double() / 127).float())
    q = torch.round((x.double() / torch.where(s == 0, torch.ones_like(s), s).double()[..., None]).float())
    return torch.where((s == 0)[..., None], torch.zeros_like(q), q).to(torch.int8), s


def runs8(x):
    b, c, n = x.shape
    runs = -(-n // RUN)
    q, s = rows8(torch.nn.functional.pad(x.float(), (0, runs * RUN - n)).reshape(b, c, runs, RUN))
    return q.reshape(b, c, runs * RUN)[..., :n].contiguous(), s


def unpacked(q, s):
    return q.double() * s.double().repeat_interleave(RUN, -1)[..., : q.shape[-1]]


# ---------------------------------------------------------------- norm

SHAPES = [(1, 1), (1, 768), (3, 255), (5, 257), (2, 512), (7, 768), (9, 1000), (4, 1001), (6, 1024), (3, 1536), (2, 2048), (3, 2049), (2, 4096), (3, 5000),
          (1, 8192), (2, 8193), (2, 16384), (1300, 768), (2100, 96), (1037, 2056)]


def norm_ref(x, r, w, eps):
    h = x.double() + (0 if r is None else r.double())
    rstd = 1 / torch.sqrt((h * h).mean(-1) + eps)
    return h, rstd, h * rstd[..., None] * w.double()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,d", SHAPES)
def test_norm_and_its_gradients(t, d, dtype):
    g = gen(d * 3 + t)
    x, r, dy, dh = (normal(g, t, d, dtype=DT[dtype]) for _ in range(4))
    w = 1 + 0.1 * normal(g, d)
    u, tiny = U[dtype], TINY[dtype]
    c = (d / 64 + 64) * E                                     # of the sums over a row: 64 lanes at least share it
    for res in (r, None):
        y, h, rstd = layers.rms_norm(x, w, residual=res, eps=1e-5)
        hr, rr, yr = norm_ref(x, res, w, 1e-5)
        assert y.dtype == h.dtype == x.dtype and rstd.dtype == torch.float32
        within(h, hr, u * hr.abs() + tiny, "h")
        within(rstd, rr, c * rr, "rstd")
        within(y, yr, (u + c) * yr.abs() + tiny, "y")
        rows, h8, rstd8 = layers.rms_norm_i8(x, w, residual=res, eps=1e-5)
        assert torch.equal(h8, h) and torch.equal(rstd8, rstd)
        top = yr.abs().amax(-1)
        within(rows.scale, top / 127, c * top / 127, "scale")
        within(rows.float(), yr, (top / 127 * (0.5 + 127 * 2 * c))[:, None].expand_as(yr), "8 bits")
        assert int(rows.q.abs().amax(-1).min()) == 127
    # the gradients, of h as it was kept
    hd, dyd, wd, z = h.double(), dy.double(), w.double(), h.double() * rstd.double()[:, None]
    gg = dyd * wd
    for back in (dh, None):
        dx, dw = layers.rms_norm_backward(dy, h, w, rstd, dh=back)
        m = (gg * z).mean(-1, keepdim=True)
        ref = (0 if back is None else back.double()) + rstd.double()[:, None] * (gg - z * m)
        size = (0 if back is None else back.double().abs()) + rstd.double()[:, None] * (gg.abs() + z.abs() * (gg * z).abs().mean(-1, keepdim=True))
        within(dx, ref, u * ref.abs() + c * size + tiny, "dx")
        within(dw, (dyd * z).sum(0), (t + 64) * E * (dyd * z).abs().sum(0), "dw")
        assert all(torch.equal(a, b) for a, b in zip((dx, dw), layers.rms_norm_backward(dy, h, w, rstd, dh=back)))


def test_norm_gradients_against_differences():
    """Central differences of sum(dy y + dh h) in 64 bits: their error is of the order of the step's square."""
    g = gen(5)
    t, d, eps, step = 3, 70, 1e-3, 1e-4
    x, r, dy, dh = (normal(g, t, d) for _ in range(4))
    w = 1 + 0.2 * normal(g, d)
    _, h, rstd = layers.rms_norm(x, w, residual=r, eps=eps)
    dx, dw = layers.rms_norm_backward(dy, h, w, rstd, dh=dh)

    def loss(x_, w_):
        h_, _, y_ = norm_ref(x_, r, w_, eps)
        return float((dy.double() * y_ + dh.double() * h_).sum())

    for i in range(0, t * d, 7):
        e = torch.zeros(t * d, dtype=torch.float64, device="cuda")
        e[i] = step
        e = e.reshape(t, d)
        assert abs((loss(x.double() + e, w) - loss(x.double() - e, w)) / (2 * step) - float(dx.flatten()[i])) < 2e-5
    for i in range(0, d, 5):
        e = torch.zeros(d, dtype=torch.float64, device="cuda")
        e[i] = step
        assert abs((loss(x, w.double() + e) - loss(x, w.double() - e)) / (2 * step) - float(dw[i])) < 2e-5


def test_norm_of_special_rows():
    """Zeros, the smallest numbers, infinities and NaN, each in a row of its own, with ordinary rows between them."""
    g = gen(1)
    x = normal(g, 9, 300)
    x[1] = 0
    x[3] = 1e-38
    x[5, 17] = float("inf")
    x[7, 299] = float("nan")
    w = torch.ones(300, device="cuda")
    y, h, rstd = layers.rms_norm(x, w, eps=1e-6)
    rows, _, _ = layers.rms_norm_i8(x, w, eps=1e-6)
    ok = [0, 1, 2, 3, 4, 6, 8]
    _, rr, yr = norm_ref(x[ok], None, w, 1e-6)
    within(y[ok], yr, 80 * E * yr.abs() + 2.0 ** -149, "ordinary rows beside others")
    within(rstd[ok], rr, 80 * E * rr)
    assert torch.isnan(y[7]).all() and torch.isnan(y[5, 17])
    assert torch.isnan(rows.scale[[5, 7]]).all() and (rows.q[[5, 7]] == 0).all()
    assert (rows.scale[[1, 3]] == 0).all() and (rows.q[[1, 3]] == 0).all() and torch.isfinite(rows.scale[ok]).all()
    # eps = 0 on a row of zeros is 0 / 0, as the formula has it
    assert torch.isnan(layers.rms_norm(torch.zeros(1, 8, device="cuda"), torch.ones(8, device="cuda"), eps=0.0)[0]).all()


@pytest.mark.parametrize("dtype", list(DT))
def test_norm_takes_slices_of_wider_rows_and_any_alignment(dtype):
    g = gen(2)
    wide, widr = normal(g, 3, 11, 900, dtype=DT[dtype]), normal(g, 3, 11, 801, dtype=DT[dtype])
    w = 1 + 0.1 * normal(g, 701)[1:]
    x, r = wide[..., 101:801], widr[..., 3:703]
    y, h, rstd = layers.rms_norm(x, w, residual=r)
    yc, hc, rc = layers.rms_norm(x.contiguous(), w, residual=r.contiguous())
    assert torch.equal(y, yc) and torch.equal(h, hc) and torch.equal(rstd, rc)
    assert all(torch.equal(a, b) for a, b in zip(layers.quantize_rows(x), layers.quantize_rows(x.contiguous())))
    dx, dw = layers.rms_norm_backward(x, h, w, rstd)
    dxc, dwc = layers.rms_norm_backward(x.contiguous(), h, w, rstd)
    assert torch.equal(dx, dxc) and torch.equal(dw, dwc)


def test_no_rows():
    w = torch.ones(64, device="cuda")
    for shape in ((0, 64), (2, 0, 64)):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        y, h, rstd = layers.rms_norm(x, w, residual=x)
        dx, dw = layers.rms_norm_backward(x, x, w, rstd)
        assert y.shape == h.shape == dx.shape == x.shape and (dw == 0).all() and layers.quantize_rows(x).q.shape == x.shape
    rows = layers.Rows8(torch.empty(0, 5, 64, dtype=torch.int8, device="cuda"), torch.empty(0, 5, device="cuda"))
    assert layers.linear_i8(rows, layers.quantize_rows(torch.ones(8, 64, device="cuda")), layout="channels", parts=2).shape == (2, 0, 4, 5)
    p = layers.act_pack(torch.empty(0, 3, 200, device="cuda"))
    assert p.scale.shape == (0, 3, 2) and layers.act_unpack(p).shape == (0, 3, 200)
    assert (layers.linear_grad_weight(torch.empty(0, 200, 7, device="cuda"), p) == 0).all()


# ---------------------------------------------------------------- 8-bit rows and products

@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("t,d", [(1, 1), (4, 31), (3, 768), (2, 3001), (1, 16384), (700, 200)])
def test_rows_in_8_bits_are_exact(t, d, dtype):
    x = normal(gen(t + d), t, d, dtype=DT[dtype])
    x[0, 0] = 100
    got, want = layers.quantize_rows(x), rows8(x)
    assert torch.equal(got.q, want[0]) and torch.equal(got.scale, want[1])


def int_rows(g, *shape):
    return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int8)


def laid_out(y, layout, parts):
    b, n, o = y.shape
    if layout == "tokens":
        return y
    y = y.reshape(b, n, parts, o // parts).permute(2, 0, 3, 1)
    return y if parts > 1 else y[0]


LINEAR = [  # b, n, k, o
    (1, 1, 1, 1), (1, 1, 64, 16), (1, 1, 777, 51), (1, 16, 4096, 48), (3, 5, 130, 33), (1, 17, 64, 64), (1, 32, 100, 40), (2, 24, 256, 96), (1, 64, 1000, 129),
    (1, 65, 64, 64), (1, 65, 63, 65), (5, 13, 48, 48), (70, 1, 80, 60), (2, 100, 129, 99), (3, 1111, 96, 192), (2, 2048, 200, 384), (1, 5000, 64, 1000),
    (1, 129, 4096, 257), (4, 4096, 768, 768), (1, 100, 8192, 300),
]


@pytest.mark.parametrize("dtype,layout,parts", [("bf16", "tokens", 1), ("bf16", "channels", 1), ("f16", "channels", 3), ("f32", "tokens", 1), ("f32", "channels", 1),
                                                ("f16", "tokens", 1)])
@pytest.mark.parametrize("b,n,k,o", LINEAR)
def test_products_in_8_bits(b, n, k, o, dtype, layout, parts):
    if o % parts:
        o += parts - o % parts
    g = gen(b + n + k + o)
    xq, wq = int_rows(g, b, n, k), int_rows(g, o, k)
    xs, ws = torch.rand(b, n, generator=g, device="cuda") + 0.01, torch.rand(o, generator=g, device="cuda") + 0.01
    bias = 100 * normal(g, o)
    sums = (xq.reshape(-1, k).double() @ wq.double().T).reshape(b, n, o) * xs.double()[..., None] * ws.double()
    for bb in (bias, None):
        y = layers.linear_i8((xq, xs), (wq, ws), bias=bb, dtype=DT[dtype], layout=layout, parts=parts)
        ref = sums + (0 if bb is None else bb.double())
        bound = U[dtype] * ref.abs() + 4 * E * (sums.abs() + bias.abs().double()) + TINY[dtype]
        within(in_range(y), in_range(laid_out(ref, layout, parts), dtype), laid_out(bound, layout, parts), "y")
    if b == 1 and layout == "tokens":
        assert torch.equal(layers.linear_i8((xq[0], xs[0]), (wq, ws), dtype=DT[dtype]), y[0])


@pytest.mark.parametrize("layout,parts,dtype", [("tokens", 1, "bf16"), ("channels", 1, "f16"), ("channels", 3, "bf16"), ("tokens", 1, "f32"), ("channels", 3, "f32")])
@pytest.mark.parametrize("b,n,k,o", [(1, 65, 4096, 4095), (5, 20, 1040, 129), (3, 100, 8192, 513), (130, 1, 2000, 99), (1, 128, 1024, 1024)])
def test_products_with_k_in_ranges(b, n, k, o, layout, parts, dtype):
    """Few tiles: k goes in ranges, the last one shorter; whole numbers, so every output is that of the sum at once."""
    if o % parts:
        o += parts - o % parts
    g = gen(b + n + k + o)
    xq, wq = int_rows(g, b, n, k), int_rows(g, o, k)
    xs, ws = torch.rand(b, n, generator=g, device="cuda") + 0.01, (torch.rand(o, generator=g, device="cuda") + 0.01) / k
    bias = normal(g, o)
    ref = (xq.reshape(-1, k).double() @ wq.double().T).reshape(b, n, o) * xs.double()[..., None] * ws.double()
    bound = (U[dtype] + 4 * E) * (ref.abs() + bias.abs().double()) + TINY[dtype]
    y = layers.linear_i8((xq, xs), (wq, ws), bias=bias, dtype=DT[dtype], layout=layout, parts=parts)
    within(y, laid_out(ref + bias.double(), layout, parts), laid_out(bound, layout, parts))
    assert torch.equal(y, layers.linear_i8((xq, xs), (wq, ws), bias=bias, dtype=DT[dtype], layout=layout, parts=parts))


@pytest.mark.parametrize("layout,parts,dtype", [("tokens", 1, "bf16"), ("channels", 1, "f16"), ("channels", 3, "bf16"), ("tokens", 1, "f32"), ("channels", 3, "f32")])
@pytest.mark.parametrize("b,n,k,o", [(33, 512, 832, 1200), (7, 2600, 64, 3840), (1, 20011, 272, 1023), (3, 8192, 16, 768), (1, 19000, 100, 900)])
def test_products_of_many_tiles(b, n, k, o, layout, parts, dtype):
    """Several tiles to a workgroup: inside y and at its ends, across sequences and parts, of one step and of many, the last one short; every
    output against the exact sums."""
    g = gen(b + n + k + o)
    xq, wq = int_rows(g, b, n, k), int_rows(g, o, k)
    xs, ws = torch.rand(b, n, generator=g, device="cuda") + 0.01, (torch.rand(o, generator=g, device="cuda") + 0.01) / k
    bias = normal(g, o)
    sums = (xq.reshape(-1, k).float() @ wq.float().T).double() if k < 1000 else (xq.reshape(-1, k).double() @ wq.double().T)   # (below 2^24: exact)
    ref = sums.reshape(b, n, o) * xs.double()[..., None] * ws.double()
    bound = (U[dtype] + 4 * E) * (ref.abs() + bias.abs().double()) + TINY[dtype]
    ref = ref + bias.double()
    y = layers.linear_i8((xq, xs), (wq, ws), bias=bias, dtype=DT[dtype], layout=layout, parts=parts)
    within(y, laid_out(ref, layout, parts), laid_out(bound, layout, parts))


def test_products_at_the_largest_sums_and_offsets():
    """All factors -128 at the largest k; y and x beyond 2^31 values; scales that are zero or NaN reach their own rows alone."""
    k = 131071
    for t in (3, 70):
        xq = torch.full((t, k), -128, dtype=torch.int8, device="cuda")
        y = layers.linear_i8((xq, torch.ones(t, device="cuda")), (xq[:2], torch.ones(2, device="cuda")), dtype=torch.float32)
        assert (y == float(np.float32(128 * 128 * k))).all()
    g = gen(3)
    for b, n, k, o in ((2, 140000, 32, 8000), (1, 150, 131008, 64), (1, 17000, 131008, 64)):
        xq, wq = int_rows(g, b, n, k), int_rows(g, o, k)
        xs, ws = torch.rand(b, n, generator=g, device="cuda"), torch.rand(o, generator=g, device="cuda")
        xs[0, 5], xs[0, 9] = 0, float("nan")
        for layout in ("tokens", "channels"):
            y = layers.linear_i8((xq, xs), (wq, ws), dtype=torch.bfloat16, layout=layout)
            y = y if layout == "tokens" else y.transpose(1, 2)
            for i, j in ((0, 0), (0, n // 2), (b - 1, n - 1), (b - 1, n - 33)):
                ref = (xq[i, j].double() @ wq.double().T) * xs[i, j].double() * ws.double()
                within(y[i, j], ref, (U["bf16"] + 4 * E) * ref.abs())
            assert (y[0, 5] == 0).all() and torch.isnan(y[0, 9]).all() and torch.isfinite(y[0, 10]).all()
            del y


# ---------------------------------------------------------------- checkpoints

ACTS = [(1, 1, 1), (1, 2, 127), (2, 3, 128), (1, 5, 129), (3, 70, 1000), (2, 64, 256), (1, 65, 1024), (2, 130, 333), (1, 1, 5001), (40, 3, 17)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("b,c,n", ACTS)
def test_checkpoints_are_exact(b, c, n, dtype):
    g = gen(b + c + n)
    x = normal(g, b, c, n, dtype=DT[dtype]) * torch.exp(2 * normal(g, b, c, 1)).to(DT[dtype])
    gate = normal(g, b, c, n, dtype=DT[dtype])
    x[0, 0, : min(n, 128)] = 0
    q, s = runs8(x)
    p = layers.act_pack(x)
    assert torch.equal(p.q, q) and torch.equal(p.scale, s)
    pt = layers.act_pack(x.transpose(1, 2).contiguous(), layout="tokens")
    assert torch.equal(pt.q, q) and torch.equal(pt.scale, s)
    pg = layers.act_pack(gate)
    for out in DT:
        back = q.float() * s.repeat_interleave(RUN, -1)[..., :n]
        assert torch.equal(layers.act_unpack(p, dtype=DT[out]), back.to(DT[out]))
        other = pg.q.float() * pg.scale.repeat_interleave(RUN, -1)[..., :n]
        assert torch.equal(layers.act_unpack(p, dtype=DT[out], gate=pg), (back * other).to(DT[out]))
    assert torch.equal(layers.act_unpack(p, dtype=DT[dtype], gate=gate), (back * gate.float()).to(DT[dtype]))
    # what is read back is within half a step
    within(layers.act_unpack(p, dtype=torch.float32), x.double(), (s * (0.5 + 127 * E)).repeat_interleave(RUN, -1)[..., :n] + x.abs() * E)


@pytest.mark.parametrize("layout", ["tokens", "channels"])
def test_checkpoints_of_special_runs(layout):
    x = normal(gen(8), 2, 66, 500)
    x[0, 3, 130:140] = float("inf")
    x[1, 65, 499] = float("nan")
    x[0, 64, :128] = 2.0 ** -101
    p = layers.act_pack(x if layout == "channels" else x.transpose(1, 2).contiguous(), layout=layout)
    back = layers.act_unpack(p, dtype=torch.float32)
    lost = torch.zeros(2, 66, 500, dtype=torch.bool, device="cuda")
    lost[0, 3, 128:256] = lost[1, 65, 384:] = True
    assert torch.equal(torch.isnan(back), lost) and (p.q[lost] == 0).all()
    assert (p.scale[0, 64, 0] == 0) and (back[0, 64, :128] == 0).all()


def test_checkpoint_beyond_32_bit_offsets():
    b, c, n = 2, 1100, 1000003
    x = torch.empty(b, c, n, dtype=torch.bfloat16, device="cuda").normal_(generator=gen(4))
    p = layers.act_pack(x)
    back = layers.act_unpack(p, dtype=torch.bfloat16)
    for i, j in ((0, 0), (0, 1099), (1, 1099), (1, 1048)):
        q, s = runs8(x[i, j][None, None])
        assert torch.equal(p.q[i, j], q[0, 0]) and torch.equal(p.scale[i, j], s[0, 0])
        assert torch.equal(back[i, j], (q.float() * s.repeat_interleave(RUN, -1)[..., :n])[0, 0].to(torch.bfloat16))


# ---------------------------------------------------------------- the weight's gradient

WEIGHT = [  # b, n, o, c
    (1, 1, 1, 1), (1, 63, 9, 5), (3, 1, 17, 33), (1, 128, 64, 64), (2, 129, 130, 127), (1, 2047, 256, 256), (5, 300, 100, 200), (2, 1000, 257, 513),
    (1, 1024, 1100, 1030), (70, 40, 33, 65), (2, 4096, 1024, 1024), (1, 640, 4100, 300),
]


def weight_check(dy, q, s, layout, dtype_dw, what=""):
    """Against the formula in 64 bits; the sums are of b n terms, with a product and a quotient for each run, and the ranges' sums."""
    b, c, n = q.shape
    x = unpacked(q, s).permute(0, 2, 1).reshape(-1, c)
    d = (dy if layout == "tokens" else dy.transpose(1, 2)).reshape(b * n, -1).double()
    ref, size = d.T @ x, d.abs().T @ x.abs()
    got = layers.linear_grad_weight(dy, (q, s), layout=layout, dtype=DT[dtype_dw])
    assert got.dtype == DT[dtype_dw]
    runs = b * -(-n // RUN)
    within(in_range(got), in_range(ref, dtype_dw), U[dtype_dw] * ref.abs() + (b * n + 4 * runs + 260) * E * size + TINY[dtype_dw], what)
    assert torch.equal(got, layers.linear_grad_weight(dy, (q, s), layout=layout, dtype=DT[dtype_dw]))
    return got


@pytest.mark.parametrize("dtype,dtype_dw", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", WEIGHT)
def test_weight_gradient(b, n, o, c, layout, dtype, dtype_dw):
    g = gen(b + n + o + c)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n) * torch.exp(2 * normal(g, b, c, 1)))
    weight_check(dy, q, s, layout, dtype_dw)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(3, 144, 520, 260), (2, 16, 264, 513), (1, 208, 1032, 1000), (70, 48, 40, 65), (2, 1040, 2304, 768), (5, 2048, 128, 128),
                                     (1, 176, 8, 1)])
def test_weight_gradient_in_pieces_of_16_bytes(b, n, o, c, layout, dtype):
    """Samples in sixteens and channels in eights: what goes straight to LDS. Half runs that end early, tiles that are mostly empty, and the same
    from tensors that start 2 bytes later, which do not."""
    g = gen(b + n + o + c)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n) * torch.exp(2 * normal(g, b, c, 1)))
    weight_check(dy, q, s, layout, "f32")
    moved = torch.empty(dy.numel() + 1, dtype=dy.dtype, device="cuda")[1:].view(dy.shape)
    weight_check(moved.copy_(dy), q, s, layout, "f32")


@pytest.mark.parametrize("n", [1200, 1201])
@pytest.mark.parametrize("layout", ["tokens", "channels"])
def test_weight_gradient_of_scales_far_apart(layout, n):
    """Runs of zeros, first, last and in a row; runs 2^90 below and above their neighbours, where dy is zero in the larger ones (what is left is
    then the small ones' sums); -128 among the values; a NaN scale, which reaches its channel alone."""
    g = gen(11)
    b, o, c = 2, 72, 140
    q, s = runs8(normal(g, b, c, n))
    q[0, 7, :40] = -128
    s[:, 1] = 0
    s[0, 2, :3] = 0
    s[1, 3, 5:] = 0
    s[0, 4, 1::2] *= 2.0 ** -90
    s[:, 5, ::2] *= 2.0 ** -45
    s[:, 6] *= 2.0 ** torch.arange(0, -200, -20, device="cuda").float()[: s.shape[-1]]
    s[0, 8, 2:] = 2.0 ** -106
    q[s.repeat_interleave(RUN, -1)[..., :n] == 0] = 0
    dy = normal(g, b, n, o)
    dy[0, 128:256] = dy[0, 384:512] = 0
    dy[0, :256, 9] = 0
    dy[1, :, 9] = 0
    for dtype in DT:
        d = dy.to(DT[dtype])
        weight_check(d if layout == "tokens" else d.transpose(1, 2).contiguous(), q, s, layout, "f32", dtype)
    s[1, 30, 4] = float("nan")
    q[1, 30, 512:640] = 0
    got = layers.linear_grad_weight(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), (q, s), layout=layout)
    assert torch.isnan(got[:, 30]).all() and int(torch.isnan(got).sum()) == o


def test_weight_gradient_against_differences():
    """The projection is linear in its weight: a central difference of sum(dy . y) in 64 bits is the derivative up to rounding."""
    g = gen(12)
    b, n, o, c = 2, 200, 5, 6
    dy, p = normal(g, b, n, o), layers.act_pack(normal(g, b, c, n))
    x = unpacked(*p)
    dw = layers.linear_grad_weight(dy, p)
    w = normal(g, o, c).double()

    def loss(w_):
        return float((dy.double() * (x.transpose(1, 2) @ w_.T)).sum())

    for i in range(o * c):
        e = torch.zeros(o * c, dtype=torch.float64, device="cuda")
        e[i] = 0.5
        e = e.reshape(o, c)
        assert abs(loss(w + e) - loss(w - e) - float(dw.flatten()[i])) < 1e-3 * 0.5


def test_weight_gradient_from_the_precomputed_product_of_a_projection():
    """What the gradient is for: the same as that of the 8-bit projection's own input, to the rounding of y."""
    g = gen(13)
    x, dy = normal(g, 2, 300, 64), normal(g, 2, 300, 32)
    p = layers.act_pack(x, layout="tokens")
    dw = layers.linear_grad_weight(dy, p)
    xa = layers.act_unpack(p, dtype=torch.float32).transpose(1, 2).reshape(-1, 64).double().requires_grad_(False)
    w = normal(g, 32, 64).double().requires_grad_(True)
    ((xa @ w.T) * dy.reshape(-1, 32).double()).sum().backward()
    within(dw, w.grad, 700 * E * (dy.reshape(-1, 32).double().abs().T @ xa.abs()))


# ---------------------------------------------------------------- streams and graphs

def all_calls(x, r, w, wq, dy, gate):
    rows, h, rstd = layers.rms_norm_i8(x, w, residual=r)
    y = layers.linear_i8(rows, wq, layout="channels", parts=2)
    p = layers.act_pack(y[0])
    u = layers.act_unpack(p, gate=layers.act_pack(gate, layout="tokens"))
    dw = layers.linear_grad_weight(dy, p, dtype=torch.float32)
    y2, h2, _ = layers.rms_norm(x, w, residual=r)
    return (h, rstd, y, u, dw, y2, *layers.rms_norm_backward(x, h2, w, rstd, dh=r))


def inputs(seed, t=333):
    g = gen(seed)
    x, r, gate, dy = (normal(g, 2, t, d, dtype=torch.bfloat16) for d in (192, 192, 96, 80))
    return x, r, 1 + 0.1 * normal(g, 192), layers.quantize_rows(normal(g, 192, 192)), dy, gate


def test_on_another_stream():
    """Inputs made on one stream, used on another that waits for it, beside work on the first."""
    want = all_calls(*inputs(1))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    args = inputs(1)
    side.wait_stream(torch.cuda.current_stream())
    noise = torch.randn(4096, 4096, device="cuda")
    for _ in range(4):
        noise = noise @ noise * 1e-3
    with torch.cuda.stream(side):
        got = all_calls(*args)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("t", [3, 333])
def test_captured_in_a_graph(t):
    args = inputs(2, t)
    all_calls(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_calls(*args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_calls(*args)
    for seed in (3, 4, 5):
        new = inputs(seed, t)
        want = all_calls(*new)
        for a, b in zip(args, new):
            for p, q in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)):
                p.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), seed

"""The operators around the convolutions on the GPU where a size, a place or a value is at the end of what a call takes. Tolerances as in
test_layers_gpu.py."""
import pytest
import torch

from paper_2311_05908_amd import fftconv, layers
from test_layers_gpu import DT, E, RUN, U, gen, int_rows, norm_ref, normal, runs8, unpacked, weight_check, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(1, 65, 1, 40), (2, 70, 1, 7), (3, 134, 1, 130), (1, 66, 2, 33), (2, 129, 3, 20), (1, 193, 2, 128), (1, 71, 1, 5), (2, 80, 3, 16)])
def test_weight_gradient_of_few_channels(b, n, o, c, layout, dtype):
    """Less than 8 channels of dy and a few samples behind a half run: the last piece of a sample reaches over several of those."""
    g = gen(b + n + o + c)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n))
    weight_check(dy, q, s, layout, "f32")
    assert torch.equal(layers.linear_grad_weight(dy, (q, s), layout=layout, dtype=DT[dtype]), layers.linear_grad_weight(dy, (q, s), layout=layout).to(DT[dtype]))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(2, 1200, 72, 140), (2, 1201, 72, 140), (1, 128, 16, 8), (3, 656, 1032, 1030), (3, 655, 1032, 1030), (1, 16, 8, 2), (1, 3, 2, 1)])
def test_weight_gradient_where_a_scale_is_zero(b, n, o, c, layout, dtype):
    """q is not zero there: a run whose scale is zero stands for zeros all the same, be it the first of a channel, one between others, the last, several,
    or all."""
    g = gen(21)
    dy = normal(g, *((b, n, o) if layout == "tokens" else (b, o, n)), dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n) * torch.exp(3 * normal(g, b, c, 1)))
    s[0, 0::6, 0] = 0
    s[-1, 1::6, -1] = 0
    s[:, 2::6, s.shape[-1] // 2] = 0
    s[:, 3::6, 1::2] = 0
    s[:, 4::12] = 0
    got = weight_check(dy, q, s, layout, "f32")
    assert c <= 4 or bool((got[:, 4::12] == 0).all())
    assert torch.equal(got, layers.linear_grad_weight(dy, (q * (s != 0).repeat_interleave(RUN, -1)[..., :n], s), layout=layout))


def check_places(y, xq, xs, wq, ws, layout, places):
    """Outputs of the tokens at these places (b, n), sixty or so before and after each, against the definition."""
    b, n, k = xq.shape
    for i, j in places:
        lo, hi = max(0, j - 60), min(n, j + 60)
        got = y[i, lo:hi] if layout == "tokens" else y[i, :, lo:hi].T
        ref = (xq[i, lo:hi].double() @ wq.double().T) * xs[i, lo:hi].double()[:, None] * ws.double()
        within(got, ref, (U["bf16"] + 4 * E) * ref.abs(), (i, j))


@pytest.mark.parametrize("layout,o", [("tokens", 3), ("channels", 2)])
def test_products_of_more_rows_than_32_bits_count_bytes_of_scales(layout, o):
    """2^30 tokens and more: the scales of those behind are theirs, not those 2^30 tokens before."""
    g = gen(61)
    n, k = (1 << 30) + 5000, 16
    xq = torch.randint(-128, 128, (1, n, k), generator=g, device="cuda", dtype=torch.int8)
    wq, ws = int_rows(g, o, k), torch.rand(o, generator=g, device="cuda") + 0.1
    xs = torch.rand(1, n, generator=g, device="cuda") + 0.1
    y = layers.linear_i8((xq, xs), (wq, ws), layout=layout)
    check_places(y, xq, xs, wq, ws, layout, [(0, j) for j in (0, 1 << 15, 1 << 29, (1 << 30) - 1, 1 << 30, (1 << 30) + 300, (1 << 30) + 2049, n - 1)])
    del xq, xs, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("b,n", [(512, 4194303), (331, 6487863)])
def test_products_of_nearly_2_31_rows(b, n):
    """2^31 - 512 tokens, the most that are taken, and 2^31 - 995, which end inside a tile; several sequences, whose ends lie inside tiles."""
    g = gen(62)
    k = 16
    xq = torch.randint(-128, 128, (b, n, k), generator=g, device="cuda", dtype=torch.int8)
    wq, ws = int_rows(g, 1, k), torch.rand(1, generator=g, device="cuda") + 0.1
    xs = torch.rand(b, n, generator=g, device="cuda") + 0.1
    y = layers.linear_i8((xq, xs), (wq, ws), layout="channels")
    check_places(y, xq, xs, wq, ws, "channels", [(i, j) for i in (0, 1, b // 2, b // 2 + 1, b - 1) for j in (0, n // 3, n - 1)])
    del xq, xs, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("layout,shape", [("channels", ((1 << 20) + 3, 513, 1)), ("tokens", ((1 << 24) + 5, 1, 64)), ("tokens", ((1 << 18) + 1, 1, 4097))])
def test_checkpoints_of_more_runs_than_a_launch_has_threads_for(layout, shape):
    """Single samples, a run each: 2^29 runs, and 2^24 tiles, are 2^32 threads and more. 127 steps of a value's own scale are the value, to bf16."""
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen(71)).abs_().clamp_(min=2.0 ** -20)
    x[::2] *= -1
    p = layers.act_pack(x, layout=layout)
    assert p.q.shape[2] == 1 and p.scale.shape == p.q.shape
    assert int(p.q.min()) == -127 and int(p.q.max()) == 127 and int((p.q == 0).sum()) == 0 and float(p.scale.min()) > 0
    back = layers.act_unpack(p)
    assert torch.equal(back.reshape(shape[0], -1), x.reshape(shape[0], -1))
    p = None
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,layout", [(1, "tokens"), (3, "channels"), (20, "tokens")])
def test_products_of_few_tokens_into_more_channels_than_a_launch_has_threads_for(t, layout):
    """From 2^27 outputs on, 512 threads for sixteen of them, a launch has 2^32 threads; k = 1."""
    g = gen(72)
    o = (1 << 27) + 77
    xq, wq = int_rows(g, 1, t, 1), int_rows(g, o, 1)
    xs, ws = torch.rand(1, t, generator=g, device="cuda") + 0.1, torch.rand(o, generator=g, device="cuda") + 0.1
    y = layers.linear_i8((xq, xs), (wq, ws), layout=layout)
    for i in range(t):
        ref = wq[:, 0].float() * float(xq[0, i, 0]) * ws * xs[0, i]
        got = (y[0, i] if layout == "tokens" else y[0, :, i]).float()
        assert bool(((got - ref).abs() <= (U["bf16"] + 8 * E) * ref.abs()).all()), i
    del y
    torch.cuda.empty_cache()


def test_products_of_nearly_2_31_rows_of_no_sixteens():
    """2^31 - 512 tokens with k = 3: 2^24 - 4 tiles of 128, a launch of nearly 2^32 threads."""
    g = gen(73)
    b, n, k = 512, 4194303, 3
    xq = torch.randint(-128, 128, (b, n, k), generator=g, device="cuda", dtype=torch.int8)
    wq, ws = int_rows(g, 1, k), torch.rand(1, generator=g, device="cuda") + 0.1
    xs = torch.rand(b, n, generator=g, device="cuda") + 0.1
    y = layers.linear_i8((xq, xs), (wq, ws), layout="channels")
    check_places(y, xq, xs, wq, ws, "channels", [(i, j) for i in (0, 1, 255, 256, 257, 510, 511) for j in (0, n // 3, n - 1)])
    del xq, xs, y
    torch.cuda.empty_cache()


def test_weight_gradient_of_no_sequences_into_more_values_than_a_launch_has_threads_for():
    """2^32 zeros, a thread for each, through the C ABI (the binding makes them itself)."""
    lib = fftconv.load()
    o, c = 1 << 16, (1 << 16) + 1
    dw = torch.ones(o, c, device="cuda")
    need = lib.fftconv_workspace_bytes_linear_grad_weight(0, 5, o, c, 1, 0)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    some = torch.zeros(16, device="cuda").data_ptr()
    assert lib.fftconv_linear_grad_weight(some, some, some, dw.data_ptr(), 0, 5, o, c, 1, 0, 0, work.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert not bool(dw.any())
    del dw, work
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", list(DT))
def test_norm_of_a_slice_goes_back_without_a_residual(dtype):
    """h is what the backward pass takes also where x is a slice of wider rows and there is no residual."""
    g = gen(31)
    wide, dy = normal(g, 3, 11, 900, dtype=DT[dtype]), normal(g, 3, 11, 700, dtype=DT[dtype])
    w = 1 + 0.1 * normal(g, 700)
    x = wide[..., 101:801]
    for norm in (layers.rms_norm, layers.rms_norm_i8):
        y, h, rstd = norm(x, w)
        yc, hc, rc = norm(x.contiguous(), w)
        assert torch.equal(h, x) and torch.equal(rstd, rc)
        assert all(torch.equal(a, b) for a, b in zip(y, yc))
        assert all(torch.equal(a, b) for a, b in zip(layers.rms_norm_backward(dy, h, w, rstd), layers.rms_norm_backward(dy, hc, w, rc)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 70, 255, 768, 1001, 2048, 4096, 5000, 8193, 16384])
def test_norm_of_rows_whose_squares_leave_fp32(d, dtype):
    """Finite rows beyond 1.8e19 and below 1e-19, next to ordinary ones, with eps from 0 up, against the formula in 64 bits: y, h, rstd, 8 bits, the
    gradients."""
    g = gen(d)
    size = torch.tensor([1.0, 1e19, 1e20, 1e30, 2.0 ** 124, 1e-19, 1e-20, 1e-25, 1e-30, 1e-37], device="cuda")
    x = (normal(g, 10, d).clamp(-7, 7) * size[:, None]).to(DT[dtype])
    x[x == 0] = 1e-37
    dy, w = normal(g, 10, d, dtype=DT[dtype]), 1 + 0.1 * normal(g, d)
    u, c = U[dtype], (d / 64 + 64) * E
    for eps in (0.0, 1e-70, 1e-50, 1e-40, 1e-30, 1e-6, 1e30):
        hr, rr, yr = norm_ref(x, None, w, eps)
        y, h, rstd = layers.rms_norm(x, w, residual=torch.zeros_like(x), eps=eps)
        assert torch.equal(h, x)
        within(rstd, rr, c * rr + 2.0 ** -149, "rstd")
        within(y, yr, (u + c) * yr.abs() + 2.0 ** (-149 if dtype == "f32" else -134), "y")
        rows, _, _ = layers.rms_norm_i8(x, w, eps=eps)
        top = yr.abs().amax(-1)
        tiny = top < 2.0 ** -99
        within(rows.scale[~tiny], top[~tiny] / 127, c * top[~tiny] / 127, "scale")
        within(rows.float()[~tiny], yr[~tiny], (top / 127 * (0.5 + 127 * 2 * c))[~tiny, None].expand_as(yr[~tiny]), "8 bits")
        # (of the rstd that the pass left, which has less than 24 bits where it is subnormal)
        z, gg, r64 = h.double() * rstd.double()[:, None], dy.double() * w.double(), rstd.double()[:, None]
        dx, dw = layers.rms_norm_backward(dy, h, w, rstd)
        ref = r64 * (gg - z * (gg * z).mean(-1, keepdim=True))
        over = ref.abs().amax(-1) > 1e38                      # (beyond the type)
        span = r64 * (gg.abs() + z.abs() * (gg * z).abs().mean(-1, keepdim=True))
        within(dx[~over], ref[~over], (u * ref.abs() + c * span + 2.0 ** (-149 if dtype == "f32" else -134))[~over], "dx")
        within(dw, (dy.double() * z).sum(0), 80 * E * (dy.double() * z).abs().sum(0), "dw")


def test_norm_of_the_smallest_and_largest_numbers():
    """Subnormal rows with eps = 0, whose rstd no fp32 number holds, and rows of fp32's largest number."""
    w = torch.ones(300, device="cuda")
    x = torch.full((4, 300), 2.0 ** -149, device="cuda")
    x[1] *= torch.arange(1, 301, device="cuda")
    x[2:] = 3.4028234e38
    x[3, ::2] *= -1
    _, _, yr = norm_ref(x, None, w, 0.0)
    y, h, rstd = layers.rms_norm(x, w, eps=0.0)
    within(y, yr, 80 * E * yr.abs())
    assert torch.isinf(rstd[:2]).all()
    # an infinity or NaN in a row is no finite row: as before
    x[0, 3], x[2, 5] = float("inf"), float("nan")
    rows, _, _ = layers.rms_norm_i8(x, w, eps=0.0)
    assert torch.isnan(rows.scale[[0, 2]]).all() and torch.isfinite(rows.scale[[1, 3]]).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("n,o,c", [(1200, 72, 140), (1201, 72, 140), (2, 1, 1), (640, 1032, 1030)])
def test_weight_gradient_of_infinities(n, o, c, layout, dtype):
    """An infinity in dy reaches its own output channel: an infinity of the product's sign, NaN where the 8-bit value is 0 or two of them cancel; NaN is
    NaN there; everything else is as without them."""
    g = gen(41)
    dy = normal(g, 1, n, o, dtype=DT[dtype])
    q, s = runs8(normal(g, 1, c, n))
    q[0, c // 2, 0] = 0
    at = {(0, 0): float("inf")}
    if o > 1:
        at.update({(n // 2, 1): float("-inf"), (n - 1, o - 1): float("nan"), (1, 9): float("inf"), (n - 2, 9): float("inf")})
    plain = dy.clone()
    for (i, j), v in at.items():
        dy[0, i, j], plain[0, i, j] = v, 0
    turned = (lambda t: t) if layout == "tokens" else (lambda t: t.transpose(1, 2).contiguous())
    got = layers.linear_grad_weight(turned(dy), (q, s), layout=layout)
    x = q[0].double() * s[0].double().repeat_interleave(RUN, -1)[..., :n]
    want = layers.linear_grad_weight(turned(plain), (q, s), layout=layout).double()
    for (i, j), v in at.items():
        want[j] += v * x[:, i]
    assert torch.equal(torch.nan_to_num(got.double(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))


@pytest.mark.parametrize("layout", ["tokens", "channels"])
def test_weight_gradient_of_the_largest_numbers(layout):
    """fp32 dy above bf16's largest number, and every other 24-bit number: no part of it is lost or an infinity."""
    g = gen(42)
    n, o, c = 130, 40, 9
    dy = torch.zeros(1, n, o, device="cuda")
    big = torch.tensor([3.4028234e38, 3.39e38, 3.3961775e38, 2.0 ** 127, -3.4028234e38, 1.1754944e-38, 1.5e-30, -1e30], device="cuda")
    dy[0, torch.arange(o, device="cuda") * 3, torch.arange(o, device="cuda")] = big.repeat(5)
    q = torch.where(torch.rand(1, c, n, generator=g, device="cuda") < 0.5, -1, 1).to(torch.int8)
    s = torch.full((1, c, 2), 0.5, device="cuda")
    got = layers.linear_grad_weight(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), (q, s), layout=layout)
    ref = dy[0].double().T @ (q[0].double().T * 0.5)
    within(got, ref, 3 * E * ref.abs() + 2.0 ** -133)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(4, 4096, 130, 200), (3, 5000, 520, 300), (4, 4096, 1152, 1030), (5, 3001, 1101, 1040), (200, 17, 64, 70)])
def test_weight_gradient_of_whole_numbers_is_exact(b, n, o, c, layout, dtype):
    """Whole numbers whose sums of magnitudes stay below 2^24, scales that are powers of two: every sum on the way is a number that fp32 holds, so the result
    is the formula's in every bit, however many terms there are and in whatever order. (Worst-case bounds grow with the terms and would let much pass.)"""
    g = gen(51)
    top = (1 << 24) // (b * n * 127)
    assert top >= 3
    dy = torch.randint(-min(top, 127), min(top, 127) + 1, (b, n, o), generator=g, device="cuda").to(DT[dtype])
    q = torch.randint(-127, 128, (b, c, n), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    s = torch.ones(b, c, -(-n // RUN), device="cuda") * 2.0 ** -torch.arange(c, device="cuda").remainder(20).float()[:, None]
    ref = dy.reshape(-1, o).double().T @ unpacked(q, s).permute(0, 2, 1).reshape(-1, c)
    got = layers.linear_grad_weight(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), (q, s), layout=layout)
    assert torch.equal(got.double(), ref)
    got = layers.linear_grad_weight(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), (q, s), layout=layout, dtype=DT[dtype])
    assert torch.equal(got, ref.to(DT[dtype]))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("b,n,o,c", [(2, 4096, 130, 200), (2, 1201, 72, 140), (2, 4096, 1152, 1030)])
def test_weight_gradient_keeps_all_bits_of_dy(b, n, o, c, layout, dtype):
    """One sample of dy to an output channel, numbers of all of the type's bits and of sizes down to its subnormal ones: a result is one product, rounded where
    its parts are added up, not more. A part of fp32's 24 bits left out would be 2^-16 of it."""
    g = gen(52)
    value = normal(g, o).to(DT[dtype])
    value[::5] *= 2.0 ** {"f16": -14, "bf16": -60, "f32": -60}[dtype]
    dy = torch.zeros(b, n, o, dtype=DT[dtype], device="cuda")
    at = torch.randint(0, b * n, (o,), generator=g, device="cuda")
    dy.reshape(-1, o)[at, torch.arange(o, device="cuda")] = value
    q = torch.randint(1, 128, (b, c, n), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    s = torch.full((b, c, -(-n // RUN)), 2.0 ** -3, device="cuda")
    ref = value.double()[:, None] * unpacked(q, s).permute(0, 2, 1).reshape(-1, c)[at]
    got = layers.linear_grad_weight(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), (q, s), layout=layout)
    within(got, ref, 3 * E * ref.abs())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["tokens", "channels"])
@pytest.mark.parametrize("n", [1200, 1201])
def test_weight_gradient_of_negative_scales(n, layout, dtype):
    """Scales that no call leaves but that the formula holds for: of either sign, 2^120 apart, so that sums in units of the smaller ones leave fp32."""
    g = gen(91)
    b, o, c = 3, 1032, 1030
    dy = normal(g, b, n, o, dtype=DT[dtype])
    q, s = runs8(normal(g, b, c, n))
    s[:, 1::4, 1::2] *= -(2.0 ** -120)
    s[:, 2::4, ::2] *= -1
    s[:, 3::4] *= -1
    s[:, 3::4, 1::2] *= 2.0 ** -120
    weight_check(dy if layout == "tokens" else dy.transpose(1, 2).contiguous(), q, s, layout, "f32")

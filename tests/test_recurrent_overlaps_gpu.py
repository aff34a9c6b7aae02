"""On the GPU: results that overlap what else a call of the recurrent layer's operators reads or writes are refused and leave everything as it was; tensors side by
side in one buffer are taken and give the bits of tensors apart."""
import pytest
import torch

from paper_2311_05908_amd import fftconv, layers

pytestmark = pytest.mark.gpu


def side_by_side(ts):
    """Copies of tensors, one where the other ends (behind a first value, so that none is aligned to more than its elements)."""
    size = ts[0].element_size()
    store = torch.empty(size + sum(t.numel() * t.element_size() for t in ts), dtype=torch.uint8, device="cuda")
    at, views = size, []
    for t in ts:
        n = t.numel() * t.element_size()
        views.append(store[at:at + n].view(t.dtype).view(t.shape).copy_(t))
        at += n
    return views


def test_step():
    g = torch.Generator(device="cuda").manual_seed(1)
    u, w, v, state = (torch.randn(7, 1001, generator=g, device="cuda") for _ in range(4))
    kept = [t.clone() for t in (u, w, v, state)]
    out = torch.empty_like(state)
    y = layers.gated_step(u, w, state, v=v, out=out)
    for t in (u, w, v):
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, state, v=v, out=t)
    both = torch.zeros(8, 1001, device="cuda")
    both[:7] = state
    for a, b in ((both[:7], both[1:]), (both[1:], both[:7])):
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, a, v=v, out=b)
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.gated_step(u, w, state, v=a, out=b)
    assert all(torch.equal(a, b) for a, b in zip((u, w, v, state), kept)) and not both[7].any()
    a, b, c, d, e = side_by_side([u, out, w, state, v])
    assert torch.equal(layers.gated_step(a, c, d, v=e, out=b), y) and torch.equal(b, out)
    assert all(torch.equal(x, k) for x, k in zip((a, c, e, d), kept))
    assert torch.equal(layers.gated_step(a, c, d, v=e), y) and torch.equal(d, out)          # in place


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,c,n", [(2, 3, 5000), (2, 24, 1001)])
def test_scans_side_by_side(b, c, n, dtype):
    """Through the C ABI, rows in segments and not: operands, results and workspace in one buffer, each where another ends."""
    g = torch.Generator(device="cuda").manual_seed(2)
    u, w, v, dy = (torch.randn(b, c, n, generator=g, device="cuda").to(dtype) for _ in range(4))
    state, dlast = (torch.randn(b, c, generator=g, device="cuda") for _ in range(2))
    lengths = torch.tensor([n, n // 2], dtype=torch.int32, device="cuda")
    y, last, kept = layers.gated_scan(u, w, v=v, state=state, lengths=lengths, keep=True)
    d, dstate = layers.gated_scan_backward(dy, u, w, kept, v=v, dlast=dlast, lengths=lengths)
    lib, code = fftconv.load(), {torch.float32: 0, torch.bfloat16: 2}[dtype]
    need = lib.fftconv_workspace_bytes_gated_scan(b, c, n, code)
    assert (need > 0) == (n == 5000)

    def buffer(*ts):
        """Stretches of one buffer for tensors (copies) and sizes in bytes, in the order given."""
        sizes = [t if isinstance(t, int) else t.numel() * t.element_size() for t in ts]
        store, at, views = torch.full((sum(sizes),), 0xff, dtype=torch.uint8, device="cuda"), 0, []
        for t, size in zip(ts, sizes):
            views.append(store[at:at + size])
            if not isinstance(t, int):
                views[-1].view(t.dtype).view(t.shape).copy_(t)
            at += size
        return views

    all_, rows = u.numel() * u.element_size(), 4 * b * c
    ws, state_, last_, u_, y_, w_, v_, kept_, lengths_ = buffer(need, state, rows, u, all_, w, v, kept.numel() * 4, lengths)
    where = [t.data_ptr() for t in (u_, w_, v_, state_, lengths_, y_, last_, kept_)]
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.fftconv_gated_scan(*where, b, c, n, 0, code, ws.data_ptr(), stream) == 0
    for got, want in ((y_, y), (last_, last), (kept_, kept), (u_, u), (w_, w), (v_, v), (state_, state), (lengths_, lengths)):
        assert torch.equal(got.view(want.dtype).view(want.shape), want)
    ws, dlast_, dstate_, dy_, du_, dw_, dv_, u_, w_, v_, kept_, lengths_ = buffer(need, dlast, rows, dy, all_, all_, all_, u, w, v, kept, lengths)
    where = [t.data_ptr() for t in (dy_, u_, w_, v_, kept_, dlast_, lengths_, du_, dw_, dv_, dstate_)]
    assert lib.fftconv_gated_scan_backward(*where, b, c, n, 0, code, ws.data_ptr(), stream) == 0
    for got, want in ((du_, d[0]), (dw_, d[1]), (dv_, d[2]), (dstate_, dstate), (dy_, dy), (u_, u), (w_, w), (v_, v), (kept_, kept), (dlast_, dlast), (lengths_, lengths)):
        assert torch.equal(got.view(want.dtype).view(want.shape), want)


def test_clipping_by_a_norm_beside_the_gradients():
    """A norm in a slot of the buffer that is written is refused and nothing changes; in the slot behind it, it is taken."""
    g = torch.Generator(device="cuda").manual_seed(3)
    flat = torch.randn(100003, generator=g, device="cuda")
    norm = layers.grad_norm([flat])
    was = flat.clone()
    ts = [flat[:60000], flat[60000:100002]]
    for at in (0, 59999, 60000, 100001):
        with pytest.raises(fftconv.FFTConvError, match="overlaps"):
            layers.clip_grads(ts, 1.0, norm=flat[at])
    other = torch.full_like(flat, 7.0)
    with pytest.raises(fftconv.FFTConvError, match="overlaps"):
        layers.clip_grads([flat], 1.0, out=[other], norm=other[5])
    assert torch.equal(flat, was) and bool((other == 7.0).all())
    flat[100002] = norm
    want = [t.clone() for t in ts]
    layers.clip_grads(want, 1.0, norm=norm)
    assert float(layers.clip_grads(ts, 1.0, norm=flat[100002])) == float(norm) == float(flat[100002])
    assert all(torch.equal(a, b) for a, b in zip(ts, want)) and not torch.equal(ts[0], was[:60000])
    # read alone, it may be anywhere
    flat.copy_(was)
    layers.clip_grads([flat], 2.0, out=[other], norm=flat[17:18].abs_())
    assert torch.equal(other[17], torch.clamp(2.0 / (flat[17].double() + 1e-6), max=1.0).float() * flat[17])

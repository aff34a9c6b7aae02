"""The norm that clipping takes and gives, on the GPU: one that comes with the call, and limits without bound."""
import ctypes

import pytest
import torch

from paper_2311_05908_amd import fftconv, layers

pytestmark = pytest.mark.gpu
F32, BF16 = 0, 2


def call(grads, out, norm_in, norm, limit=1.0):
    """fftconv_clip_grads of fp32 tensors through the C ABI."""
    lib, n = fftconv.load(), len(grads)
    pointers = lambda ts: (ctypes.c_int64 * max(1, n))(*(t.data_ptr() for t in ts))  # noqa: E731
    counts, types = (ctypes.c_int64 * max(1, n))(*(t.numel() for t in grads)), (ctypes.c_int * max(1, n))(*([F32] * n))
    ws = torch.empty(lib.fftconv_workspace_bytes_clip_grads(counts, n), dtype=torch.uint8, device="cuda")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    rc = lib.fftconv_clip_grads(pointers(grads), None if out is None else pointers(out), counts, types, None, n, limit, 1e-6, ptr(norm_in), ptr(norm), ptr(ws),
                                torch.cuda.current_stream().cuda_stream)
    assert rc == 0, lib.fftconv_last_error()


@pytest.mark.parametrize("sizes", [[5], [3, 70000, 1], [100] * 300, [9000000], [0, 0], []], ids=lambda s: "%d tensors of %d" % (len(s), sum(s)))
def test_the_norm_goes_where_the_call_says(sizes):
    """The gradients' own, with results and without, and one that came with the call: whatever was there before."""
    g = torch.Generator(device="cuda").manual_seed(len(sizes))
    grads = [torch.randn(s, generator=g, device="cuda") for s in sizes]
    want = layers.grad_norm(grads)
    out = [torch.empty_like(t) for t in grads]
    given = torch.full((), 12.5, device="cuda")
    for results, norm_in in ((None, None), (out, None), (out, given)):
        norm = torch.full((), -1.0, device="cuda")
        call(grads, results, norm_in, norm)
        assert float(norm) == float(want if norm_in is None else given)
    call(grads, out, given, given)                            # (the same place: as it was)
    assert float(given) == 12.5
    for t, o in zip(grads, out):
        assert torch.equal(o, t * torch.tensor(1.0 / (12.5 + 1e-6), device="cuda", dtype=torch.float64).float())


def test_limits_without_bound():
    """A limit of infinity clips nothing, whatever the norm: c = 1, and only what is NaN makes everything NaN. (Its quotient by an infinite norm is no number.)"""
    inf, nan = float("inf"), float("nan")
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for bad in (None, inf, -inf, nan):
            grads = [torch.arange(-50.0, 50.0, device="cuda").to(dtype), torch.ones(9000, device="cuda", dtype=dtype)]
            if bad is not None:
                grads[1][8999] = bad
            out = [torch.empty_like(t) for t in grads]
            norm = layers.clip_grads(grads, inf, out=out)
            inside = [t.clone() for t in grads]
            assert torch.equal(layers.clip_grads(inside, inf).nan_to_num(nan=-1.0), norm.nan_to_num(nan=-1.0))
            for ts in (out, inside):
                if bad is nan or bad != bad:
                    assert torch.isnan(norm) and all(torch.isnan(t).all() for t in ts)
                else:
                    assert all(torch.equal(a, b) for a, b in zip(ts, grads))
            assert bad is None or bad != bad or torch.isinf(norm)
    # an infinite norm and a limit that is one: nothing but zeros, and NaN where the infinity was
    t = torch.tensor([3.0, inf], device="cuda")
    assert torch.isinf(layers.clip_grads([t], 3e38)) and t[0] == 0 and torch.isnan(t[1])


@pytest.mark.parametrize("into", [True, False])
def test_a_norm_that_comes_with_the_call_is_taken_and_returned(into):
    """Not the gradients' own: the factor is that of the given one, which comes back as it was, the same tensor; gradients change only in place."""
    g = torch.Generator(device="cuda").manual_seed(9)
    grads = [torch.randn(s, generator=g, device="cuda") for s in (4097, 12, 70001)]
    was = [t.clone() for t in grads]
    own = float(layers.grad_norm(grads))
    given = torch.full((), 4 * own, device="cuda")
    out = [torch.empty_like(t) for t in grads] if into else None
    back = layers.clip_grads(grads, own, out=out, norm=given)
    assert back is given and float(given) == float(torch.tensor(4 * own))
    factor = torch.tensor(own / (float(given) + 1e-6), dtype=torch.float64).float().cuda()
    for t, w in zip(out if into else grads, was):
        assert torch.equal(t, w * factor)
    if into:
        assert all(torch.equal(a, b) for a, b in zip(grads, was))


def test_results_elsewhere_leave_the_gradients_alone():
    t = torch.tensor([3.0, 4.0], device="cuda")
    out = torch.empty(2, device="cuda")
    for limit, eps in ((5.0, 0.0), (2.5, 0.0), (0.0, 1e-6), (float("inf"), 1e-6), (1e-30, 1e-6)):
        layers.clip_grads([t], limit, out=[out], eps=eps)
        assert t.tolist() == [3.0, 4.0]

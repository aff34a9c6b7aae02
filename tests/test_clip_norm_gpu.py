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

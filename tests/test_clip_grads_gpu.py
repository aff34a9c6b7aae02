"""The gradients' norm and their clipping on the GPU, against their definitions in 64 bits.

Squares of fp32 numbers are within 2^-53 of themselves in 64 bits and so is every addition: with a billion of them the norm is within 2^-24 of itself
(half a step of fp32, rounded at the end), and so are the factor and each product; results in 16 bits are rounded once more."""
import pytest
import torch

from paper_2311_05908_amd import fftconv, layers

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
E = 2.0 ** -24


def grads(sizes, dtypes, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(size * torch.randn(s, generator=g, device="cuda")).to(DT[dtypes[i % len(dtypes)]]) for i, s in enumerate(sizes)]


def norm64(ts):
    return float(sum(float(t.double().square().sum()) for t in ts) ** 0.5)


def check(got, ts, norm, limit, eps=1e-6):
    c = min(1.0, limit / (norm + eps))
    for y, t in zip(got, ts):
        want = t.double() * c
        assert y.shape == t.shape
        bound = (4 * E + U[y.dtype]) * want.abs() + (2.0 ** -25 if y.dtype == torch.float16 else 2.0 ** -149)
        assert y.numel() == 0 or bool(((y.double() - want).abs() <= bound).all())


SETS = [[1], [768], [8191, 8192, 8193], [3, 0, 5], [(64, 64), (7,), (3, 5, 11), (100000,)], [1] * 300, [1000003, 17], [(257, 129)] * 130]


@pytest.mark.parametrize("limited", [True, False])
@pytest.mark.parametrize("dtypes", [("f32",), ("bf16",), ("f16",), ("f32", "bf16", "f16")])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%d tensors" % len(s))
def test_norm_and_clipping(sizes, dtypes, limited):
    ts = grads(sizes, dtypes)
    norm = norm64(ts)
    limit = norm * (0.37 if limited else 2.0)
    got = layers.grad_norm(ts)
    assert got.shape == () and got.dtype == torch.float32 and abs(float(got) - norm) <= 2 * E * norm
    same, wide = [torch.full_like(t, 7) for t in ts], [torch.full_like(t, 7, dtype=torch.float32) for t in ts]
    for out in (same, wide):
        again = layers.clip_grads(ts, limit, out=out)
        assert torch.equal(again, got)
        check(out, ts, norm, limit)
    inside = [t.clone() for t in ts]
    layers.clip_grads(inside, limit)
    assert all(torch.equal(a, b) for a, b in zip(inside, same))
    if not limited:
        assert all(torch.equal(a, b) for a, b in zip(inside, ts))
    given = [t.clone() for t in ts]
    assert layers.clip_grads(given, limit, norm=2 * got) is not None
    check(given, ts, 2 * float(got), limit)


def test_tensors_at_any_element_beside_others():
    """Views of one buffer, one behind the other: what lies between them stays."""
    for dtype in DT.values():
        store = torch.randn(5000, device="cuda").to(dtype)
        was = store.clone()
        ts = [store[1:8], store[9:1010], store[1010:1011], store[1013:4999]]
        norm = norm64(ts)
        layers.clip_grads(ts, norm / 3)
        check(ts, [was[1:8], was[9:1010], was[1010:1011], was[1013:4999]], norm, norm / 3)
        for i in (0, 8, 1011, 1012, 4999):
            assert store[i] == was[i]


def test_squares_beyond_fp32():
    for value, dtype in ((1e30, torch.float32), (1e-30, torch.float32), (3e38, torch.bfloat16), (1e-40, torch.float32), (6e-8, torch.float16)):
        t = torch.full((1000,), value, device="cuda").to(dtype)
        norm = float(t[0].double()) * 1000 ** 0.5
        got = float(layers.grad_norm([t]))
        assert abs(got - norm) <= 2 * E * norm + 2.0 ** -149 or (norm > 3.4e38 and got == float("inf"))
        out = torch.empty(1000, device="cuda")
        layers.clip_grads([t], 1.0, out=[out])
        check([out], [t], norm, 1.0)


def test_what_is_not_a_number():
    for bad in (float("nan"), float("inf")):
        ts = grads([100, 20000], ("f32",))
        ts[1][12345] = bad
        was = [t.clone() for t in ts]
        norm = layers.clip_grads(ts, 1.0)
        if bad != bad:
            assert torch.isnan(norm) and all(torch.isnan(t).all() for t in ts)
        else:
            assert torch.isinf(norm) and not ts[0].any() and torch.isnan(ts[1][12345]) and int(torch.isnan(ts[1]).sum()) == 1
        assert float(layers.grad_norm(was[:1])) > 0


def test_edges_of_the_limit():
    t = torch.tensor([3.0, 4.0], device="cuda")
    assert torch.equal(t, torch.tensor([3.0, 4.0], device="cuda"))
    out = torch.empty(2, device="cuda")
    assert float(layers.clip_grads([t], 5.0, out=[out], eps=0.0)) == 5.0 and torch.equal(out, t)
    layers.clip_grads([t], 2.5, out=[out], eps=0.0)
    assert torch.equal(out, t / 2)
    layers.clip_grads([t], 0.0, out=[out])
    assert not out.any()
    layers.clip_grads([t], float("inf"), out=[out])
    assert torch.equal(out, t)
    zero = torch.zeros(9, device="cuda")
    assert float(layers.clip_grads([zero], 1.0, eps=0.0)) == 0 and not zero.any()
    assert float(layers.grad_norm([])) == 0 and float(layers.clip_grads([], 1.0)) == 0
    assert float(layers.grad_norm([torch.empty(0, device="cuda")])) == 0
    assert float(layers.grad_norm([t, t])) == pytest.approx(50 ** 0.5, rel=2 * E)        # (read twice, counted twice)


def test_a_billion_values():
    """Beyond 2^32 bytes; every value the same, so that the norm is known."""
    n = (1 << 31) + 12345
    t = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    norm = 0.5 * n ** 0.5
    assert abs(float(layers.clip_grads([t], norm / 4)) - norm) <= 2 * E * norm
    want = float(torch.tensor(0.5 * 0.25).bfloat16())
    assert bool((t[-20000:] == want).all()) and bool((t[:20000] == want).all()) and int((t != want).sum()) == 0


def test_streams_and_graphs():
    """Two graphs with a workspace each, replayed over new gradients with eager calls between."""
    sizes = [768, (64, 100), 30000, 5]
    made = [grads(sizes, ("bf16", "f32"), seed=s, size=2.0 ** s) for s in range(3)]
    limit = norm64(made[1])

    def eager(ts):
        out = [torch.empty_like(t) for t in ts]
        return layers.clip_grads(ts, limit, out=out), out

    want = [eager(ts) for ts in made]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm, out = eager(made[2])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(norm, want[2][0]) and all(torch.equal(a, b) for a, b in zip(out, want[2][1]))
    ins = [[t.clone() for t in made[s]] for s in (0, 1)]
    graphs, norms = [], []
    for ts in ins:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norms.append(layers.clip_grads(ts, limit))
        graphs.append(graph)
    for turn in range(4):
        for i, ts in enumerate(ins):
            for a, b in zip(ts, made[(turn + i) % 3]):
                a.copy_(b)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        eager(made[turn % 3])
        for i, ts in enumerate(ins):
            norm, out = want[(turn + i) % 3]
            assert torch.equal(norms[i], norm) and all(torch.equal(a, b) for a, b in zip(ts, out))


def test_refusals():
    t, u = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    for a, kw in (([t.cpu()], {}), ([t[::2]], {}), ([t.int()], {}), ([t], dict(out=[])), ([t], dict(out=[u.half()])), ([t], dict(out=[u[:5]])),
                  ([t], dict(norm=torch.ones(2, device="cuda"))), ([t], dict(norm=torch.ones(())))):
        with pytest.raises(ValueError):
            layers.clip_grads(a, 1.0, **kw)
    both = torch.ones(20, device="cuda")
    for a, kw in (([t, t], {}), ([both[:12], both[8:]], {}), ([t, u], dict(out=[u, t])), ([t, u], dict(out=[both[:10], both[5:15]])),
                  ([both[:10]], dict(out=[both[5:15]])), ([t], dict(max_norm=-1.0)), ([t], dict(max_norm=float("nan"))), ([t], dict(max_norm=0.0, eps=0.0)),
                  ([t], dict(eps=-1.0))):
        with pytest.raises(fftconv.FFTConvError):
            layers.clip_grads(a, **{"max_norm": 1.0, **kw})
    layers.clip_grads([t, t], 1.0, out=[both[:10], both[10:]])

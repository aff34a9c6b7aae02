"""How far a projection from e4m3 with long rows may be from its value, closely enough that a part of k that is left out shows.

With block sums B_j of exact products (magnitudes: M_j), scales s_j, their product rounded as the operator says, and c_j = s_j B_j, y = sum of c_j. Off are
  a block's sum of 128 products in fp32 on the matrix cores, in whatever order, an addition off by up to a unit in the last place, 2 E: 256 E M_j;
  for 16-bit results what products of e4m3 lose: in the eight neighbours along k the largest power of two of a product, with the operands' exponents added,
      is 2^e; every product keeps its multiple of 2^(e - 13) and loses the rest, L_j over a block;
  the total over blocks in fp32, one multiply-add after the other along runs of consecutive blocks, the runs' sums after one another: E of what was added up each
      time, and that is the sum of some consecutive c_j, at most the distance R between the largest and the smallest of the sums c_0 + ... + c_j (and 0), so
      2 blocks E R; once more 2^-10 of that for what is itself off in it;
  the result, rounded to its type: U.
E = 2^-24."""
import torch

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F8 = torch.float8_e4m3fn


def rows8(x):
    """Rows (t, k), k a multiple of 16, in e4m3 and their scales (blocks, t)."""
    t, k = x.shape
    blocks = -(-k // 128)
    x = torch.nn.functional.pad(x, (0, blocks * 128 - k)).view(t, blocks, 128)
    s = x.abs().amax(-1) / torch.full((), 448.0, device=x.device)
    return (x / s[..., None]).view(t, -1)[:, :k].to(F8), s.t().contiguous()


def block_sums(rows, weight):
    """(s_j B_j, s_j M_j, s_j L_j), each (t, o, blocks) in 64 bits."""
    (xq, xs), (wq, ws) = rows, weight
    (t, k), o, blocks = xq.shape, wq.shape[0], xs.shape[0]
    pad = lambda q: torch.nn.functional.pad(q.float(), (0, blocks * 128 - k)).view(q.shape[0], blocks, 16, 8)  # noqa: E731
    power = lambda q: torch.frexp(q.abs().clamp(min=2.0 ** -6))[1]  # noqa: E731       (of a number below 2^-6: the least there is)
    x, w = pad(xq), pad(wq)
    ex, ew = power(x), power(w)
    out = torch.empty(3, t, o, blocks, dtype=torch.float64, device=xq.device)
    step = max(1, (1 << 26) // (t * o * 128))
    for j in range(0, blocks, step):
        at = slice(j, min(j + step, blocks))
        p = x[:, None, at] * w[None, :, at]                     # eight bits of significand: exact in fp32
        top = (ex[:, None, at] + ew[None, :, at]).amax(-1, keepdim=True) - 2
        lost = torch.fmod(p, torch.ldexp(torch.ones_like(p[..., :1]), top - 13))
        for i, v in enumerate((p, p.abs(), lost.abs())):
            out[i, :, :, at] = v.double().sum((-1, -2))
    s = xs.t()[:, None] * ws.repeat_interleave(128, 0)[None, :o]       # (t, o, blocks), rounded to fp32
    return out * s.double()


def value_and_bound(sums, dtype):
    """y and how far from it a result may be, both (t, o) in 64 bits."""
    c, m, lost = sums
    y = c.sum(-1)
    runs = torch.nn.functional.pad(c.cumsum(-1), (1, 0))
    r = runs.amax(-1) - runs.amin(-1)
    bound = 256 * E * m.sum(-1) + 2 * c.shape[-1] * E * r * (1 + 2.0 ** -10)
    if dtype != torch.float32:
        bound = bound + lost.sum(-1)
    return y, bound * (1 + U[dtype]) + U[dtype] * y.abs()


def operands(t, k, o, device, seed):
    """Rows with some channels twenty times as large, and a weight that keeps their size."""
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=device)  # noqa: E731
    x = normal(t, k) * (1 + 19 * (torch.rand(k, generator=g, device=device) < 0.02))
    w, blocks = normal(o, k) / k ** 0.5, -(-k // 128)
    big = torch.nn.functional.pad(w, (0, blocks * 128 - k)).abs().view(o, blocks, 128).amax(-1)
    ws = torch.stack([part.amax(0) for part in big.split(128)]) / torch.full((), 448.0, device=device)
    return rows8(x), ((w / ws.repeat_interleave(128, 0)[:o].repeat_interleave(128, 1)[:, :k]).to(F8), ws)


# Few and many tokens whose products go by ranges of k; tokens, k, outputs.
LONG = [(1, 1 << 20, 40), (40, (1 << 18) + 16, 33), (70, (1 << 18) + 80, 130), (65, 16384, 100), (1, 32768, 40), (17, 16384 + 48, 200), (300, 4096, 512)]

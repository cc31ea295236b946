"""The block's operators where element and byte offsets pass 32 bits, checked on rows from all over."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -23


def _room(gib):
    if torch.cuda.get_device_properties(0).total_memory < gib * 2 ** 30:
        pytest.skip("too little memory")


def _randn(rows, cols, seed, std=1.0):
    """bf16, made a few thousand rows at a time."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    for part in out.split(max(1, (1 << 26) // cols)):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(std))
    return out


@pytest.fixture()
def ctx():
    c = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    yield c
    c.close()
    torch.cuda.empty_cache()


def test_norms(ctx):
    _room(64)
    t, h = 140001, 16384                                     # 2.3e9 elements
    x, y = _randn(t, h, 1), _randn(t, h, 2, 3.0)
    wp, wn = _randn(1, h, 3)[0], _randn(1, h, 4)[0]
    xo, n, r1, r2 = torch.empty_like(x), torch.empty_like(x), torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    ctx.block_norm_forward(x, y, wp, None, wn, xo, n, r1, r2, scale=0.5)
    rows = torch.tensor([0, 1, 65536, 131071, 131072, t - 2, t - 1], device="cuda")
    x64, y64 = x[rows].double(), y[rows].double()
    s1 = torch.rsqrt((y64 ** 2).mean(1, keepdim=True) + 1e-6)
    x1 = x64 + 0.5 * y64 * s1 * wp.double()
    want = x1 * torch.rsqrt((x1 ** 2).mean(1, keepdim=True) + 1e-6) * wn.double()
    tol = 100 * UNIT + 2.0 ** -8
    assert bool(((xo[rows].double() - x1).abs() <= tol * (x64.abs() + (x1 - x64).abs()).clamp_min(1e-6)).all())
    assert float((n[rows].double() - want).norm() / want.norm()) < 2.0 ** -8
    ctx.reserve_block_norm(t, h)
    dw = [torch.empty_like(wp), torch.empty_like(wn)]
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    ctx.block_norm_backward(x, y, xo, y, wp, None, wn, r1, r2, dx, dy, dw[0], None, dw[1], scale=0.5)
    xh = xo[rows].double() * r2[rows].double()[:, None]
    u = y64 * wn.double()
    d = x64 + r2[rows].double()[:, None] * (u - xh * (u * xh).mean(1, keepdim=True))
    assert float((dx[rows].double() - d).norm() / d.norm()) < 2.0 ** -8


def test_gradients(ctx):
    _room(32)
    g = _randn(70001, 65536, 5, 1e-3)                         # 4.6e9 elements
    nc = torch.zeros(2, device="cuda")
    ctx.grad_sumsq_batch([edgc.Tensor(g, g)])
    ctx.clip_batch([edgc.Tensor(g, g)], 1e6, nc)              # clips nothing
    want = math.sqrt(math.fsum(float((p.double() ** 2).sum()) for p in g.split(2048)))
    assert abs(float(nc[0]) - want) <= 4 * UNIT * want and float(nc[1]) == 1.0
    rows = [0, 1, 32767, 65535, 65536, 70000]
    before = g[rows].clone()
    ctx.clip_batch([edgc.Tensor(g, g)], 1.0, nc)
    coef = min(1.0, 1.0 / (want + 1e-6))
    assert bool(((g[rows].double() - before.double() * coef).abs() <= 2.0 ** -8 * before.double().abs() * coef).all())


def test_feed_forward(ctx):
    _room(96)
    t, h, f = 36992, 64, 65536                                # projections of 2.4e9 elements
    x, dy = _randn(t, h, 6), _randn(t, h, 7, 1e-2)
    wg, wu, wd = _randn(f, h, 8, h ** -0.5), _randn(f, h, 9, h ** -0.5), _randn(h, f, 10, f ** -0.5)
    w = edgc.FeedForward(wg, wu, wd)
    ctx.reserve_ff(torch.bfloat16, t, h, f, backward=True)
    y = torch.empty_like(x)
    gate, up = (torch.empty(t, f, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ctx.ff_forward(w, x, y, gate, up)
    dx, dwg, dwu, dwd = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)
    ctx.ff_backward(w, x, gate, up, dy, dx, dwg, dwu, dwd)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    rows = torch.tensor([0, 31, 32767, 32768, t - 1], device="cuda")
    X, G, U, D = x[rows].double(), gate[rows].double(), up[rows].double(), dy[rows].double()
    assert rel(gate[rows], X @ wg.double().t()) < 2.0 ** -8 and rel(up[rows], X @ wu.double().t()) < 2.0 ** -8
    s = torch.sigmoid(G)
    a, da = G * s, s * (1 + G * (1 - s))
    # two roundings to bf16 in the norm: of an intermediate operand and of the result
    assert rel(y[rows], (a * U) @ wd.double().t()) < 2.0 ** -7
    dA = D @ wd.double()
    assert rel(dx[rows], (dA * U * da) @ wg.double() + (dA * a) @ wu.double()) < 2.0 ** -7
    cols = torch.tensor([0, 1, 40000, f - 1], device="cuda")
    G, U, dA = gate[:, cols].double(), up[:, cols].double(), dy.double() @ wd[:, cols].double()
    s = torch.sigmoid(G)
    assert rel(dwg[cols], (dA * U * s * (1 + G * (1 - s))).t() @ x.double()) < 2.0 ** -7
    assert rel(dwu[cols], (dA * G * s).t() @ x.double()) < 2.0 ** -7
    assert rel(dwd[:, cols], dy.double().t() @ (G * s * U)) < 2.0 ** -7

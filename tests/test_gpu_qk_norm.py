"""The norms of queries and keys with the rotation by position, and their gradients, against 64-bit arithmetic on the host."""
import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    c = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    yield c
    c.close()


def randn(shape, seed, dtype, std=1.0, mean=0.0):
    return (mean + std * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype)


def frequencies(rot):
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))


def swap(x, n, interleaved):
    """Each rotated dimension's partner, and its sign in the rotation; 0 for the others."""
    y, sign = torch.zeros_like(x), torch.zeros(x.shape[-1], dtype=torch.float64)
    if interleaved:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = x[..., 1:2 * n:2], x[..., 0:2 * n:2]
        sign[0:2 * n:2], sign[1:2 * n:2] = -1, 1
    else:
        y[..., :n], y[..., n:2 * n] = x[..., n:2 * n], x[..., :n]
        sign[:n], sign[n:2 * n] = -1, 1
    return y, sign


def angles(positions, inv_freq, dim, interleaved):
    """Cosine and sine of every dimension of a head: tokens x 1 x dim."""
    t, n = len(positions), len(inv_freq)
    a = positions.double()[:, None] * inv_freq
    c, s = torch.ones(t, 1, dim, dtype=torch.float64), torch.zeros(t, 1, dim, dtype=torch.float64)
    for k in range(2):
        at = slice(k, 2 * n, 2) if interleaved else slice(k * n, (k + 1) * n)
        c[:, 0, at], s[:, 0, at] = torch.cos(a), torch.sin(a)
    return c, s


def rotate(x, cos, sin, n, interleaved):
    y, sign = swap(x, n, interleaved)
    return x * cos + y * sin * sign


def want_forward(x, w, cos, sin, n, interleaved):
    x, w = x.double(), w.double()
    z = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    # sizes of both terms that an output is the sum of
    return rotate(z, cos, sin, n, interleaved), z.abs() + swap(z.abs(), n, interleaved)[0]


def fp32(dim):
    """Relative to the terms of an output: sine and cosine to two units of 2^-23 and the rounding of their angle, three products and a sum, root and reciprocal;
    the sum of dim squares, by lanes of up to 16 elements and across them, halved by the root."""
    return 2.0 ** -21 + (8 + min(dim, 16) + 6) / 2 * 2.0 ** -24


def check_forward(got, x, w, cos, sin, n, interleaved):
    want, size = want_forward(x, w, cos, sin, n, interleaved)
    bound = size * fp32(x.shape[-1]) + want.abs() * torch.finfo(got.dtype).eps / 2 + 1e-40
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


def check_backward(dx, dw, dy, x, w, cos, sin, n, interleaved):
    dim = x.shape[-1]
    leaf_x, leaf_w = x.double().requires_grad_(), w.double().requires_grad_()
    r = (leaf_x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = rotate(leaf_x * r * leaf_w, cos, sin, n, interleaved)
    want_x, want_w = torch.autograd.grad(y, (leaf_x, leaf_w), dy.double())
    r, xh = r.detach(), (leaf_x * r).detach()
    a = dy.double().abs()
    d = a + swap(a, n, interleaved)[0]                      # what the gradient before the rotation is at most
    u = d * w.double().abs()
    # (the mean's fp32 sum is of dim products)
    size = r * (u + xh.abs() * (u * xh.abs()).mean(-1, keepdim=True)) * 3
    err = (dx.double().cpu() - want_x).abs()
    bound = size * (fp32(dim) + (min(dim, 16) + 6) * 2.0 ** -24) + want_x.abs() * torch.finfo(dx.dtype).eps / 2 + 1e-40
    assert bool((err <= bound).all()), float((err / bound).max())
    # the weights': sums of tokens x heads products, one after the other at worst
    size = (d * xh.abs()).sum((0, 1))
    err = (dw.double().cpu() - want_w).abs()
    bound = size * (fp32(dim) + x.shape[0] * x.shape[1] * 2.0 ** -24) + want_w.abs() * torch.finfo(dw.dtype).eps / 2 + 1e-40
    assert bool((err <= bound).all()), float((err / bound).max())


def layout(t, kind, value):
    """Queries or keys on the GPU as one of the layouts they come in: (buffer, view)."""
    n, h, d = t.shape
    if kind == "dense":
        wide = torch.full((n, h, d), value, dtype=t.dtype, device="cuda")
        view = wide
    elif kind == "packed":                                  # columns of a wider row
        wide = torch.full((n, h * d + 13), value, dtype=t.dtype, device="cuda")
        view = wide[:, 5:5 + h * d].view(n, h, d) if n == 1 else wide[:, 5:5 + h * d].unflatten(1, (h, d))
    elif kind == "heads":                                   # a head's tokens together
        wide = torch.full((h, n + 3, d), value, dtype=t.dtype, device="cuda")
        view = wide[:, 2:2 + n].transpose(0, 1)
    else:                                                   # heads further apart than they are long
        wide = torch.full((n, h, d + 3), value, dtype=t.dtype, device="cuda")
        view = wide[..., 1:1 + d]
    view.copy_(t)
    return wide, view


CASES = [  # tokens, heads of queries and keys, dim, rotated, layout
    (1, 1, 1, 2, 2, "dense"), (1, 32, 8, 128, 128, "packed"), (3, 7, 3, 72, 40, "packed"), (8, 5, 5, 64, 64, "heads"), (9, 4, 2, 80, 80, "apart"),
    (17, 2, 0, 96, 48, "dense"), (200, 3, 1, 32, 32, "packed"), (33, 6, 2, 256, 64, "heads"), (20, 2, 1, 512, 512, "dense"), (21, 3, 2, 1, 0, "dense"),
    (10, 2, 2, 7, 6, "apart"), (64, 9, 3, 36, 18, "packed"), (11, 1, 1, 257, 256, "dense"), (5, 70, 1, 16, 16, "dense"), (2100, 2, 1, 8, 8, "packed"),
    (40, 4, 4, 192, 96, "heads"),
]


def inputs(case, dtype, positions_type=torch.int64, far=3000):
    t, hq, hk, dim, rot, kind = case
    q, k = randn((t, hq, dim), 1, dtype, 2.0), randn((t, hk, dim), 2, dtype, 0.5) if hk else None
    w_q, w_k = randn((dim,), 3, dtype, 0.2, 1.0), randn((dim,), 4, dtype, 0.2, 1.0) if hk else None
    g = torch.Generator().manual_seed(5)
    pos = torch.randint(-far, far, (t,), generator=g).to(positions_type)
    return q, k, w_q, w_k, pos, frequencies(rot)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(ctx, case, interleaved, dtype):
    t, hq, hk, dim, rot, kind = case
    q, k, w_q, w_k, pos, f = inputs(case, dtype, torch.int32 if t % 2 else torch.int64)
    cuda = lambda x: None if x is None else x.cuda()
    _, vq = layout(q, kind, 3.0)
    vk = layout(k, kind, 3.0)[1] if hk else None
    wide, out_q = layout(torch.zeros_like(q), "apart" if kind == "dense" else kind, 7.0)
    out_k = layout(torch.zeros_like(k), kind, 7.0)[1] if hk else None
    ctx.qk_norm_forward(vq, vk, cuda(w_q), cuda(w_k), cuda(pos) if rot else None, cuda(f) if rot else None, out_q, out_k, eps=EPS, interleaved=interleaved)
    cos, sin = angles(pos, f, dim, interleaved)
    check_forward(out_q, q, w_q, cos, sin, rot // 2, interleaved)
    if hk:
        check_forward(out_k, k, w_k, cos, sin, rot // 2, interleaved)
    assert torch.equal(vq.cpu(), q)
    if kind == "dense":
        assert bool((wide[..., 0] == 7.0).all()) and bool((wide[..., 1 + dim:] == 7.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(ctx, case, interleaved, dtype):
    t, hq, hk, dim, rot, kind = case
    q, k, w_q, w_k, pos, f = inputs(case, dtype)
    dq_out, dk_out = randn((t, hq, dim), 6, dtype), randn((t, hk, dim), 7, dtype) if hk else None
    cuda = lambda x: None if x is None else x.cuda()
    at = lambda x, value: layout(x, kind, value)[1] if x is not None else None
    dq, dk = at(torch.zeros_like(q), 7.0), at(torch.zeros_like(k) if hk else None, 7.0)
    dw_q, dw_k = torch.full((dim,), 9.0, dtype=dtype, device="cuda"), torch.full((dim,), 9.0, dtype=dtype, device="cuda") if hk else None
    ctx.reserve_qk_norm(t, hq, hk, dim)
    ctx.qk_norm_backward(at(dq_out, 3.0), at(dk_out, 3.0), at(q, 3.0), at(k, 3.0), cuda(w_q), cuda(w_k), cuda(pos) if rot else None, cuda(f) if rot else None,
                         dq, dk, dw_q, dw_k, eps=EPS, interleaved=interleaved)
    cos, sin = angles(pos, f, dim, interleaved)
    check_backward(dq, dw_q, dq_out, q, w_q, cos, sin, rot // 2, interleaved)
    if hk:
        check_backward(dk, dw_k, dk_out, k, w_k, cos, sin, rot // 2, interleaved)


@pytest.mark.parametrize("hk", [0, 2])
@pytest.mark.parametrize("t", [255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2049, 9000])
def test_tokens_where_the_blocks_are_dealt_out_otherwise(ctx, t, hk):
    """Few tokens have blocks of queries and of keys, more have blocks of both, of one token or several."""
    case = (t, 3, hk, 16, 8, "dense")
    q, k, w_q, w_k, pos, f = inputs(case, F32)
    dq_out, dk_out = randn((t, 3, 16), 6, F32), randn((t, hk, 16), 7, F32) if hk else None
    cuda = lambda x: None if x is None else x.cuda()
    like = lambda x: None if x is None else torch.full_like(x, 7.0, device="cuda")
    out_q, out_k, dq, dk, dw_q, dw_k = like(q), like(k), like(q), like(k), like(w_q), like(w_k)
    ctx.reserve_qk_norm(t, 3, hk, 16)
    ctx.qk_norm_forward(cuda(q), cuda(k), cuda(w_q), cuda(w_k), cuda(pos), cuda(f), out_q, out_k, eps=EPS)
    ctx.qk_norm_backward(cuda(dq_out), cuda(dk_out), cuda(q), cuda(k), cuda(w_q), cuda(w_k), cuda(pos), cuda(f), dq, dk, dw_q, dw_k, eps=EPS)
    cos, sin = angles(pos, f, 16, False)
    check_forward(out_q, q, w_q, cos, sin, 4, False)
    check_backward(dq, dw_q, dq_out, q, w_q, cos, sin, 4, False)
    if hk:
        check_forward(out_k, k, w_k, cos, sin, 4, False)
        check_backward(dk, dw_k, dk_out, k, w_k, cos, sin, 4, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rot", [0, 512])
def test_what_is_larger_than_the_caches(ctx, rot, dtype):
    """More than 2^27 bytes go past the caches: the same bits as a part of the tokens at a time, and the weights' gradients by the formulas."""
    t, hq, hk, dim = (9500 if dtype is BF16 else 4750), 6, 2, 512
    g = torch.Generator(device="cuda").manual_seed(3)
    make = lambda h: torch.randn((t, h, dim), generator=g, device="cuda").to(dtype)
    q, k, dq_out, dk_out = make(hq), make(hk), make(hq), make(hk)
    w_q, w_k = [(1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dtype) for _ in range(2)]
    pos = torch.randint(0, 5000, (t,), generator=g, device="cuda") if rot else None
    f = frequencies(rot).cuda() if rot else None
    ctx.reserve_qk_norm(t, hq, hk, dim)

    def run(at):
        some = lambda x: x[at].contiguous()
        out = [torch.full_like(some(x), 7.0) for x in (q, k, q, k)]
        dw = [torch.empty(dim, dtype=dtype, device="cuda") for _ in range(2)]
        p = pos[at].contiguous() if rot else None
        ctx.qk_norm_forward(some(q), some(k), w_q, w_k, p, f, out[0], out[1], eps=EPS)
        ctx.qk_norm_backward(some(dq_out), some(dk_out), some(q), some(k), w_q, w_k, p, f, out[2], out[3], *dw, eps=EPS)
        return out, dw

    whole, dw = run(slice(0, t))
    parts = [run(slice(i, min(i + 2000, t)))[0] for i in range(0, t, 2000)]
    for i, x in enumerate(whole):
        assert torch.equal(x, torch.cat([p[i] for p in parts]))
    if rot:
        return
    for got, x, dy in ((dw[0], q, dq_out), (dw[1], k, dk_out)):
        x, dy = x.double(), dy.double()
        terms = dy * x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        want = terms.sum((0, 1))
        bound = terms.abs().sum((0, 1)) * (fp32(dim) + t * x.shape[1] * 2.0 ** -24) + want.abs() * torch.finfo(dtype).eps / 2
        assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("far", [1 << 20, 1 << 31, 1 << 40])
def test_far_positions(ctx, far):
    """Angles of a position are as exact as their product in 64 bits, far beyond what 32 bits or one double's digits of a circle hold."""
    case = (50, 2, 1, 64, 64, "dense")
    q, k, w_q, w_k, pos, f = inputs(case, F32, far=far)
    pos[0], pos[1] = far, -far
    out_q, out_k = torch.empty_like(q).cuda(), torch.empty_like(k).cuda()
    ctx.qk_norm_forward(q.cuda(), k.cuda(), w_q.cuda(), w_k.cuda(), pos.cuda(), f.cuda(), out_q, out_k)
    cos, sin = angles(pos, f, 64, False)
    check_forward(out_q, q, w_q, cos, sin, 32, False)
    check_forward(out_k, k, w_k, cos, sin, 32, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_into_a_cache(ctx, dtype):
    """Queries over themselves; keys of one token per text into their places of a cache; the backward pass over either of its inputs."""
    case = (6, 8, 2, 64, 64, "dense")
    q, k, w_q, w_k, pos, f = inputs(case, dtype)
    qd = q.cuda()
    cache = torch.full((6, 2, 10, 64), 5.0, dtype=dtype, device="cuda")
    ctx.qk_norm_forward(qd, k.cuda(), w_q.cuda(), w_k.cuda(), pos.cuda(), f.cuda(), qd, cache[:, :, 4])
    cos, sin = angles(pos, f, 64, False)
    check_forward(qd, q, w_q, cos, sin, 32, False)
    check_forward(cache[:, :, 4], k, w_k, cos, sin, 32, False)
    assert bool((cache[:, :, :4] == 5.0).all()) and bool((cache[:, :, 5:] == 5.0).all())
    dq_out, dk_out = randn(q.shape, 6, dtype), randn(k.shape, 7, dtype)
    dq, dk = dq_out.cuda(), k.cuda()
    dw_q, dw_k = torch.empty(64, dtype=dtype, device="cuda"), torch.empty(64, dtype=dtype, device="cuda")
    ctx.reserve_qk_norm(6, 8, 2, 64)
    ctx.qk_norm_backward(dq, dk_out.cuda(), q.cuda(), dk, w_q.cuda(), w_k.cuda(), pos.cuda(), f.cuda(), dq, dk, dw_q, dw_k)
    check_backward(dq, dw_q, dq_out, q, w_q, cos, sin, 32, False)
    check_backward(dk, dw_k, dk_out, k, w_k, cos, sin, 32, False)


def test_gradients_by_differences(ctx):
    """The backward pass is that of the forward pass that runs: a loss's differences along directions, in fp32."""
    case = (12, 3, 2, 32, 24, "dense")
    q, k, w_q, w_k, pos, f = (None if x is None else x.cuda() for x in inputs(case, F32))
    c_q, c_k = randn(q.shape, 8, F32).cuda(), randn(k.shape, 9, F32).cuda()

    def loss(q, k, w_q, w_k):
        a, b = torch.empty_like(q), torch.empty_like(k)
        ctx.qk_norm_forward(q, k, w_q, w_k, pos, f, a, b)
        return float((a.double() * c_q).sum() + (b.double() * c_k).sum())
    grads = [torch.empty_like(x) for x in (q, k, w_q, w_k)]
    ctx.reserve_qk_norm(12, 3, 2, 32)
    ctx.qk_norm_backward(c_q, c_k, q, k, w_q, w_k, pos, f, *grads)
    for i in range(4):
        at = [q, k, w_q, w_k]
        way = randn(at[i].shape, 20 + i, F32).cuda()
        # third differences of size h^2 |way|^3, and 2^-22 of the outputs' sum over h, each below 2e-3 of the sizes at hand
        h = 2.0 ** -7
        plus, minus = [a + h * way if j == i else a for j, a in enumerate(at)], [a - h * way if j == i else a for j, a in enumerate(at)]
        slope, want = (loss(*plus) - loss(*minus)) / (2 * h), float((grads[i].double() * way).sum())
        size = float((grads[i].double() * way).norm()) + 1.0
        assert abs(slope - want) <= 2e-2 * size, (i, slope, want)


def test_zero_heads_and_what_is_not_finite(ctx):
    """A head of zeros stays zeros; one with NaN or Inf is its own affair."""
    q, w = randn((4, 3, 64), 1, F32), torch.ones(64)
    q[0, 0], q[1, 1, 5], q[2, 2, 7] = 0.0, float("nan"), float("inf")
    out = torch.empty_like(q).cuda()
    ctx.qk_norm_forward(q.cuda(), None, w.cuda(), None, torch.arange(4).cuda(), frequencies(64).cuda(), out, None)
    out = out.cpu()
    assert bool((out[0, 0] == 0).all())
    fine = torch.ones(4, 3, dtype=torch.bool)
    fine[1, 1] = fine[2, 2] = False
    assert bool(torch.isfinite(out[fine]).all()) and bool(torch.isnan(out[1, 1]).any()) and bool(torch.isnan(out[2, 2]).any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_tokens(ctx, dtype):
    q, w = torch.zeros(0, 3, 64, dtype=dtype, device="cuda"), torch.ones(64, dtype=dtype, device="cuda")
    dw = [torch.full((64,), 4.0, dtype=dtype, device="cuda") for _ in range(2)]
    pos, f = torch.zeros(0, dtype=torch.int64, device="cuda"), frequencies(64).cuda()
    ctx.qk_norm_forward(q, q, w, w, pos, f, q, q)
    ctx.qk_norm_backward(q, q, q, q, w, w, pos, f, q, q, *dw)
    assert all(bool((d == 0).all()) for d in dw)


def test_rows_beyond_32_bit_offsets(ctx):
    """Heads that lie 2^32 elements and more into their buffer."""
    wide = torch.zeros((3, 1 << 31), dtype=BF16, device="cuda")
    q = wide[:, 100:100 + 4 * 32].unflatten(1, (4, 32))
    x = randn((3, 4, 32), 1, BF16)
    q.copy_(x)
    w, pos, f = randn((32,), 3, BF16, 0.2, 1.0), torch.tensor([5, 6, 7]), frequencies(32)
    ctx.qk_norm_forward(q, None, w.cuda(), None, pos.cuda(), f.cuda(), q, None)
    check_forward(q, x, w, *angles(pos, f, 32, False), 16, False)
    assert int((wide != 0).sum()) <= 3 * 4 * 32


def test_the_same_call_gives_the_same_bits_also_from_a_graph(ctx):
    case = (700, 6, 2, 128, 128, "dense")
    q, k, w_q, w_k, pos, f = (x.cuda() for x in inputs(case, BF16))
    dy_q, dy_k = randn(q.shape, 6, BF16).cuda(), randn(k.shape, 7, BF16).cuda()
    outs = [torch.empty_like(x) for x in (q, k, q, k, w_q, w_k)]
    ctx.reserve_qk_norm(700, 6, 2, 128)

    def go():
        ctx.qk_norm_forward(q, k, w_q, w_k, pos, f, outs[0], outs[1])
        ctx.qk_norm_backward(dy_q, dy_k, q, k, w_q, w_k, pos, f, *outs[2:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for s in (1, 2, 1):
        q.copy_(randn(q.shape, s + 30, BF16))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outs]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))


def test_refusals(ctx):
    q, k, w, pos, f = torch.zeros(4, 3, 64, device="cuda"), torch.zeros(4, 2, 64, device="cuda"), torch.ones(64, device="cuda"), torch.arange(4).cuda(), frequencies(64).cuda()

    def refused(match, f_, *a, **kw):
        with pytest.raises(edgc.EdgcError, match=match) as e:
            f_(*a, **kw)
        assert e.value.code == -1
    for eps in (-1.0, float("nan"), float("inf")):
        refused("eps", ctx.qk_norm_forward, q, k, w, w, pos, f, q, k, eps=eps)
    refused("rotated", ctx.qk_norm_forward, q, k, w, w, pos, frequencies(66).cuda(), q, k)
    refused("overlap", ctx.qk_norm_forward, q, k, w, w, pos, f, q[:1].expand(4, 3, 64), k)
    refused("overlap", ctx.qk_norm_forward, q, k, w, w, pos, f, q, torch.zeros(64 * 5, device="cuda").as_strided((4, 2, 64), (64, 64, 1)))
    wide = torch.zeros(4, 3, 600, device="cuda")
    refused("dimensions", ctx.qk_norm_forward, wide, None, torch.zeros(600, device="cuda"), None, None, None, wide, None)
    ctx.reserve_qk_norm(3, 3, 2, 64)
    refused("reserve_qk_norm", ctx.qk_norm_backward, q, k, q, k, w, w, pos, f, q.clone(), k.clone(), w.clone(), w.clone())
    ctx.reserve_qk_norm(4, 2, 2, 64)
    refused("reserve_qk_norm", ctx.qk_norm_backward, q, k, q, k, w, w, pos, f, q.clone(), k.clone(), w.clone(), w.clone())
    refused("heads", ctx.reserve_qk_norm, 4, 0, 2, 64)
    refused("dimensions", ctx.reserve_qk_norm, 4, 1, 2, 513)

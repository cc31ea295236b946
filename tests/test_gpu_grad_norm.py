"""The global gradient norm and clipping, element by element against 64-bit arithmetic on the host."""
import math

import numpy as np
import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu

# one rounding of the product of an element and the coefficient (itself rounded to fp32): relative, per element
TOL = {torch.float32: 2.0 ** -23 + 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
# the norm is a sum of 64 bits rounded to fp32 once, the coefficient likewise
NORM_TOL = 2.0 ** -23


def _grads(shapes, dtype, seed=0, scale=1e-2):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * scale * (1 + i % 3)).to(dtype) for i, s in enumerate(shapes)]


def _host(grads, max_norm):
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    return norm, (min(1.0, max_norm / (norm + 1e-6)) if math.isfinite(norm) else 1.0)


def _check(host, outs, norm_coef, max_norm):
    norm, coef = _host(host, max_norm)
    got = norm_coef.cpu().double()
    assert abs(float(got[0]) - norm) <= NORM_TOL * norm and abs(float(got[1]) - coef) <= NORM_TOL * coef
    for h, o in zip(host, outs):
        want, o = h.double() * coef, o.cpu()
        assert o.dtype == h.dtype and o.shape == h.shape
        err = (o.double() - want).abs()
        assert bool((err <= TOL[h.dtype] * want.abs() + 1e-45).all()), float((err / want.abs().clamp_min(1e-30)).max())


SHAPES = [
    [(1,)], [(7,)], [(1, 1)], [(2047,)], [(2049,)], [(16384, 3)], [(3, 16385)],
    [(512, 512), (512,), (1,), (37, 41), (8191,), (64, 1)],
    [(33, 65)] * 64, [(5, 9)] * 65, [(129,)] * 200,
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("max_norm", [0.05, 1e6])
def test_norm_and_clipping(shapes, dtype, max_norm):
    host = _grads(shapes, dtype)
    dev = [h.cuda() for h in host]
    outs = [torch.full_like(d, 7.0) for d in dev]
    nc = torch.zeros(2, device="cuda")
    batch = edgc.PreparedBatch([edgc.Tensor(a, b) for a, b in zip(dev, outs)])
    ctx().grad_sumsq_batch(batch)
    ctx().clip_batch(batch, max_norm, nc)
    _check(host, outs, nc, max_norm)
    assert all(torch.equal(d.cpu(), h) for d, h in zip(dev, host))          # the inputs are only read


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [0.05, 1e6])
def test_in_place_and_strided_rows(dtype, max_norm):
    """Gradients that are columns of wider buffers, in place and between two strides; what lies beside them is not touched."""
    host = _grads([(70, 130), (1, 50), (513, 7), (3, 4097)], dtype, seed=3)
    wide = [torch.full((h.shape[0], h.shape[1] + 9), 5.0, dtype=dtype, device="cuda") for h in host]
    for w, h in zip(wide, host):
        w[:, 2:2 + h.shape[1]] = h.cuda()
    views = [w[:, 2:2 + h.shape[1]] for w, h in zip(wide, host)]
    to = [torch.full((h.shape[0], h.shape[1] + 5), 6.0, dtype=dtype, device="cuda") for h in host]
    tov = [w[:, 1:1 + h.shape[1]] for w, h in zip(to, host)]
    nc = torch.zeros(2, device="cuda")
    ts = [edgc.Tensor(a, b) for a, b in zip(views, tov)]
    ctx().grad_sumsq_batch(ts)
    ctx().clip_batch(ts, max_norm, nc)
    _check(host, tov, nc, max_norm)
    ts = [edgc.Tensor(a, a) for a in views]
    ctx().grad_sumsq_batch(ts)
    ctx().clip_batch(ts, max_norm, nc)
    _check(host, views, nc, max_norm)
    for w, h in zip(wide, host):
        assert bool((w[:, :2] == 5).all()) and bool((w[:, 2 + h.shape[1]:] == 5).all())
    for w, h in zip(to, host):
        assert bool((w[:, :1] == 6).all()) and bool((w[:, 1 + h.shape[1]:] == 6).all())


def test_lists_of_both_dtypes_and_a_sum_of_the_callers_own():
    a, b = _grads([(100, 100), (77,)], torch.float32, 1), _grads([(64, 65)], torch.bfloat16, 2)
    da, db = [x.cuda() for x in a], [x.cuda() for x in b]
    s = torch.full((1,), 3.0, dtype=torch.float64, device="cuda")
    nc = torch.zeros(2, device="cuda")
    ta, tb = [edgc.Tensor(x, x) for x in da], [edgc.Tensor(x, x) for x in db]
    ctx().grad_sumsq_batch(ta, s)
    ctx().grad_sumsq_batch(tb, s, accumulate=True)
    want = math.fsum(float((x.double() ** 2).sum()) for x in a + b)
    assert abs(float(s) - want) <= 1e-12 * want
    ctx().clip_batch(ta, 0.1, nc, sumsq=s)
    ctx().clip_batch(tb, 0.1, nc, sumsq=s)
    _check(a + b, da + db, nc, 0.1)
    ctx().grad_sumsq_batch([], s, accumulate=True)
    assert abs(float(s) - want) <= 1e-12 * want
    ctx().grad_sumsq_batch([], s)
    assert float(s) == 0.0
    ctx().clip_batch([], 1.0, nc, sumsq=s)
    assert nc.tolist() == [0.0, 1.0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_squares_beyond_fp32(dtype):
    """Elements whose squares overflow or vanish in 32 bits."""
    for scale in (1e25, 1e-28):
        host = [(g / g.float().abs().max().to(g.dtype) * scale).to(dtype) for g in _grads([(300, 70)], dtype, 5)]
        dev = [h.cuda() for h in host]
        nc = torch.zeros(2, device="cuda")
        s = torch.zeros(1, dtype=torch.float64, device="cuda")
        ts = [edgc.Tensor(d, torch.empty_like(d)) for d in dev]
        ctx().grad_sumsq_batch(ts, s)
        want = float((host[0].double() ** 2).sum())
        assert abs(float(s) - want) <= 1e-12 * want
        ctx().clip_batch(ts, 1.0, nc, sumsq=s)
        _check(host, [t.grad_out for t in ts], nc, 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_clips_nothing(dtype, bad):
    host = _grads([(40, 50), (9,)], dtype, 7)
    host[0][3, 4] = bad
    dev = [h.cuda() for h in host]
    nc = torch.zeros(2, device="cuda")
    ts = [edgc.Tensor(d, torch.empty_like(d)) for d in dev]
    ctx().grad_sumsq_batch(ts)
    ctx().clip_batch(ts, 0.01, nc)
    assert not math.isfinite(float(nc[0])) and float(nc[1]) == 1.0
    for h, t in zip(host, ts):
        assert torch.equal(torch.nan_to_num(h.float(), 1.0, 2.0, 3.0), torch.nan_to_num(t.grad_out.cpu().float(), 1.0, 2.0, 3.0))


def test_zero_gradients_and_the_same_bits_every_time():
    z = torch.zeros(1000, device="cuda")
    nc = torch.full((2,), 9.0, device="cuda")
    ctx().grad_sumsq_batch([edgc.Tensor(z, z)])
    ctx().clip_batch([edgc.Tensor(z, z)], 1.0, nc)
    assert nc.tolist() == [0.0, 1.0] and not z.any()
    g = torch.randn(3_000_001, device="cuda")
    s = torch.zeros(4, dtype=torch.float64, device="cuda")
    for k in range(4):
        ctx().grad_sumsq_batch([edgc.Tensor(g, g)], s[k:k + 1])
    assert len(set(s.tolist())) == 1


def test_on_another_stream():
    host = _grads([(1000, 1000)], torch.float32, 9)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        d = host[0].cuda()
        o, nc = torch.empty_like(d), torch.zeros(2, device="cuda")
        ctx().grad_sumsq_batch([edgc.Tensor(d, o)])
        ctx().clip_batch([edgc.Tensor(d, o)], 0.5, nc)
    side.synchronize()
    _check(host, [o], nc, 0.5)


def test_refusals():
    c = ctx()
    g = torch.zeros((4, 8), device="cuda")
    t = [edgc.Tensor(g, g)]
    for bad in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(edgc.EdgcError):
            c.clip_batch(t, bad)
    with pytest.raises(edgc.EdgcError):
        c.clip_batch([edgc.Tensor(g, None)], 1.0)
    with pytest.raises(edgc.EdgcError):
        c.grad_sumsq_batch([edgc.Tensor(torch.zeros((0, 8), device="cuda"), g)])
    with pytest.raises(TypeError):
        c.grad_sumsq_batch([edgc.Tensor(g.half(), g)])
    with pytest.raises(TypeError):
        c.grad_sumsq_batch([edgc.Tensor(g, g), edgc.Tensor(g.bfloat16(), g)])
    with pytest.raises(TypeError):
        c.grad_sumsq_batch(t, torch.zeros(1, device="cuda"))
    with pytest.raises(TypeError):
        c.clip_batch(t, 1.0, torch.zeros(2, device="cuda", dtype=torch.float64))

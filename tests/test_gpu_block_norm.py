"""The norms before and after a block with its gate and residual scale, forward and backward, against 64-bit arithmetic."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu

EPS = 1e-6
# fp32 arithmetic on a row of h: sums of h terms lose about sqrt(h) half-units in the mean and never more than h; a hundred units
# cover every row here.  A bf16 output adds its rounding: neighbours are 2^-7 of their size apart, half of that is 2^-8.
# Sums over t tokens of terms of either sign are held against the sum of the terms' absolute values.
UNIT = 2.0 ** -23
TOL = {torch.float32: 100 * UNIT, torch.bfloat16: 100 * UNIT + 2.0 ** -8}


def _inputs(t, h, dtype, groups, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std=1.0, mean=0.0: (mean + std * torch.randn(*s, generator=g)).to(dtype)
    d = dict(x=r(t, h), y=r(t, h, std=3.0), w_post=r(h, std=0.1, mean=1.0), w_pre=r(h, std=0.1, mean=1.0),
             gate=r(groups, h) if groups else None, dx_out=r(t, h, std=1e-2), dn=r(t, h, std=1e-2))
    return d


def _forward64(d, rows, scale, post=True, pre=True):
    d = {k: None if v is None else v.double() for k, v in d.items()}
    t, h = d["x"].shape
    x1, r1, r2, n = d["x"], None, None, None
    if post:
        gate = 1.0 if d["gate"] is None else d["gate"][torch.arange(t) // rows]
        r1 = 1 / torch.sqrt((d["y"] ** 2).mean(1) + EPS)
        x1 = d["x"] + scale * gate * d["y"] * r1[:, None] * d["w_post"]
    if pre:
        r2 = 1 / torch.sqrt((x1 ** 2).mean(1) + EPS)
        n = x1 * r2[:, None] * d["w_pre"]
    return x1, n, r1, r2


def _close(got, want, scale=None):
    """Element by element, relative to `scale` (default: the rms of the row or vector, or the element where that is larger)."""
    got, dt = got.cpu(), got.dtype
    if scale is None:
        scale = torch.maximum(want.abs(), (want ** 2).mean(-1, keepdim=True).sqrt())
    err = (got.double() - want).abs() / scale.clamp_min(1e-30)
    assert bool((err <= (TOL[dt] if dt in TOL else TOL[torch.float32])).all()), float(err.max())


def _dev(d):
    return {k: None if v is None else v.cuda() for k, v in d.items()}


SIZES = [(1, 1), (1, 4096), (2, 3), (3, 7), (5, 64), (4, 511), (9, 512), (7, 513), (33, 1000), (17, 1024), (6, 1025), (5, 2047),
         (300, 256), (70, 5120), (3, 8192), (3, 8193), (2, 16384), (2500, 96), (1100, 1536)]
GATES = ["none", "one", "token", "few"]


def _rows(gates, t):
    return {"none": 0, "one": t, "token": 1, "few": max(1, t // 3)}[gates]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h", SIZES)
@pytest.mark.parametrize("gates", GATES)
def test_forward(t, h, dtype, gates):
    rows = _rows(gates, t)
    d = _inputs(t, h, dtype, -(-t // rows) if rows else 0)
    v = _dev(d)
    xo, n = torch.full_like(v["x"], 7.0), torch.full_like(v["x"], 7.0)
    r1, r2 = torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
    ctx().block_norm_forward(v["x"], v["y"], v["w_post"], v["gate"], v["w_pre"], xo, n, r1, r2, scale=0.7, eps=EPS, rows_per_gate=rows)
    x1, n1, s1, s2 = _forward64(d, rows, 0.7)
    # x_out can cancel: against the size of its two terms
    _close(xo, x1, (d["x"].double().abs() + (x1 - d["x"].double()).abs()).clamp_min(1e-6))
    big = (d["x"].double().abs() + (x1 - d["x"].double()).abs()) * s2[:, None] * d["w_pre"].double().abs()
    _close(n, n1, torch.maximum(big, (n1 ** 2).mean(-1, keepdim=True).sqrt()))
    _close(r1, s1, s1)
    _close(r2, s2, s2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h", SIZES)
@pytest.mark.parametrize("gates", GATES)
def test_backward(t, h, dtype, gates):
    rows = _rows(gates, t)
    groups = -(-t // rows) if rows else 0
    d = _inputs(t, h, dtype, groups, seed=1)
    scale = 0.7
    x1, _, r1, r2 = _forward64(d, rows, scale)
    x1 = x1.to(dtype)
    r1, r2 = r1.float(), r2.float()
    v = _dev(d)
    dx, dy = torch.full_like(v["x"], 7.0), torch.full_like(v["x"], 7.0)
    dwp, dwn = torch.full_like(v["w_pre"], 7.0), torch.full_like(v["w_pre"], 7.0)
    dg = torch.full_like(v["gate"], 7.0) if rows else None
    ctx().reserve_block_norm(t, h)
    ctx().block_norm_backward(v["dx_out"], v["dn"], x1.cuda(), v["y"], v["w_post"], v["gate"], v["w_pre"], r1.cuda(), r2.cuda(),
                              dx, dy, dwp, dg, dwn, scale=scale, rows_per_gate=rows)
    q = {k: None if a is None else a.double() for k, a in d.items()}
    xh, yh = x1.double() * r2.double()[:, None], q["y"] * r1.double()[:, None]
    u = q["dn"] * q["w_pre"]
    D = q["dx_out"] + r2.double()[:, None] * (u - xh * (u * xh).mean(1, keepdim=True))
    gate = q["gate"][torch.arange(t) // rows] if rows else torch.ones_like(D)
    vv = scale * gate * q["w_post"] * D
    size = lambda z: torch.maximum(z.abs(), (z ** 2).mean(1, keepdim=True).sqrt())
    dsize = q["dx_out"].abs() + r2.double()[:, None] * (u.abs() + xh.abs() * (u * xh).abs().mean(1, keepdim=True))
    _close(dx, D, torch.maximum(size(D), dsize))
    vs = scale * gate.abs() * q["w_post"].abs() * dsize
    _close(dy, r1.double()[:, None] * (vv - yh * (vv * yh).mean(1, keepdim=True)),
           r1.double()[:, None] * (size(vs) + yh.abs() * (vs * yh.abs()).mean(1, keepdim=True)))
    _close(dwn, (q["dn"] * xh).sum(0), (q["dn"] * xh).abs().sum(0))
    _close(dwp, (scale * gate * D * yh).sum(0), (scale * gate.abs() * dsize * yh.abs()).sum(0))
    if rows:
        per, pers = scale * q["w_post"] * D * yh, scale * q["w_post"].abs() * dsize * yh.abs()
        idx = torch.arange(t) // rows
        zero = torch.zeros(groups, h, dtype=torch.float64)
        _close(dg, zero.index_add(0, idx, per), zero.index_add(0, idx, pers))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h", [(5, 200), (9, 1536)])
def test_each_norm_alone(t, h, dtype):
    d = _inputs(t, h, dtype, 1)
    v = _dev(d)
    o = lambda: torch.full_like(v["x"], 7.0)
    c = ctx()
    c.reserve_block_norm(t, h)
    # before the first block: n alone, then with a copy of x
    n, xo, r2 = o(), o(), torch.zeros(t, device="cuda")
    c.block_norm_forward(v["x"], None, None, None, v["w_pre"], None, n, None, r2)
    x1, n1, _, s2 = _forward64(d, 0, 1.0, post=False)
    _close(n, n1)
    c.block_norm_forward(v["x"], None, None, None, v["w_pre"], xo, n, None, r2)
    assert torch.equal(xo, v["x"])
    dx, dw = o(), torch.full_like(v["w_pre"], 7.0)
    c.block_norm_backward(None, v["dn"], v["x"], None, None, None, v["w_pre"], None, r2, dx, None, None, None, dw)
    xh, u = x1 * s2[:, None], d["dn"].double() * d["w_pre"].double()
    want = s2[:, None] * (u - xh * (u * xh).mean(1, keepdim=True))
    _close(dx, want)
    _close(dw, (d["dn"].double() * xh).sum(0), (d["dn"].double() * xh).abs().sum(0))
    # after the last block: x_out alone
    xo, r1 = o(), torch.zeros(t, device="cuda")
    c.block_norm_forward(v["x"], v["y"], v["w_post"], v["gate"], None, xo, None, r1, None, scale=0.5, rows_per_gate=t)
    x1, _, s1, _ = _forward64(d, t, 0.5, pre=False)
    _close(xo, x1, d["x"].double().abs() + (x1 - d["x"].double()).abs() + 1e-6)
    dx, dy, dwp, dg = o(), o(), torch.full_like(v["w_pre"], 7.0), torch.full_like(v["gate"], 7.0)
    c.block_norm_backward(v["dx_out"], None, None, v["y"], v["w_post"], v["gate"], None, r1, None, dx, dy, dwp, dg, None, scale=0.5,
                          rows_per_gate=t)
    assert torch.equal(dx, v["dx_out"])
    yh = d["y"].double() * s1[:, None]
    S = (d["dx_out"].double() * yh).sum(0)
    Sa = (d["dx_out"].double() * yh).abs().sum(0)
    _close(dg[0], 0.5 * d["w_post"].double() * S, 0.5 * d["w_post"].double().abs() * Sa)
    _close(dwp, 0.5 * d["gate"][0].double() * S, 0.5 * d["gate"][0].double().abs() * Sa)


def test_gradients_are_the_differences_of_the_forward_pass():
    """The backward pass in fp32 along random directions against central differences of the 64-bit forward pass."""
    t, h, rows, scale = 6, 160, 4, 0.6
    d = {k: None if v is None else v.float() for k, v in _inputs(t, h, torch.float32, 2, seed=4).items()}
    loss = lambda q: float((q["dx_out"].double() * _forward64(q, rows, scale)[0]).sum() + (q["dn"].double() * _forward64(q, rows, scale)[1]).sum())
    x1, _, r1, r2 = _forward64(d, rows, scale)
    v = _dev(d)
    out = {"x": torch.empty_like(v["x"]), "y": torch.empty_like(v["y"]), "w_post": torch.empty_like(v["w_post"]),
           "gate": torch.empty_like(v["gate"]), "w_pre": torch.empty_like(v["w_pre"])}
    ctx().reserve_block_norm(t, h)
    ctx().block_norm_backward(v["dx_out"], v["dn"], x1.float().cuda(), v["y"], v["w_post"], v["gate"], v["w_pre"], r1.float().cuda(),
                              r2.float().cuda(), out["x"], out["y"], out["w_post"], out["gate"], out["w_pre"], scale=scale,
                              rows_per_gate=rows)
    g = torch.Generator().manual_seed(8)
    for k, grad in out.items():
        e = torch.randn(d[k].shape, generator=g, dtype=torch.float64)
        step = 1e-5
        up, dn = dict(d), dict(d)
        up[k], dn[k] = d[k].double() + step * e, d[k].double() - step * e
        diff = (loss(up) - loss(dn)) / (2 * step)
        got = float((grad.cpu().double() * e).sum())
        size = float((grad.cpu().double() * e).abs().sum())
        # the gradient's fp32 arithmetic against the sum of its terms, and the differences' step^2 and 64-bit cancellation
        assert abs(got - diff) <= 100 * UNIT * size + 1e-6 * size, (k, got, diff)


def test_buffers_in_place_and_no_tokens():
    t, h = 40, 2000
    d = _inputs(t, h, torch.float32, 1, seed=2)
    v, c = _dev(d), ctx()
    c.reserve_block_norm(t, h)
    n, xo, r1, r2 = torch.empty_like(v["x"]), torch.empty_like(v["x"]), torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    args = dict(scale=0.5, rows_per_gate=t)
    c.block_norm_forward(v["x"], v["y"], v["w_post"], v["gate"], v["w_pre"], xo, n, r1, r2, **args)
    x, y = v["x"].clone(), v["y"].clone()
    c.block_norm_forward(x, y, v["w_post"], v["gate"], v["w_pre"], x, y, r1, r2, **args)
    assert torch.equal(x, xo) and torch.equal(y, n)
    grads = lambda: [torch.empty_like(v[k]) for k in ("w_post", "gate", "w_pre")]
    a, b = grads(), grads()
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    c.block_norm_backward(v["dx_out"], v["dn"], xo, v["y"], v["w_post"], v["gate"], v["w_pre"], r1, r2, dx, dy, a[0], a[1], a[2], **args)
    dxi, dni = v["dx_out"].clone(), v["dn"].clone()
    c.block_norm_backward(dxi, dni, xo, v["y"], v["w_post"], v["gate"], v["w_pre"], r1, r2, dxi, dni, b[0], b[1], b[2], **args)
    assert torch.equal(dxi, dx) and torch.equal(dni, dy) and all(torch.equal(p, q) for p, q in zip(a, b))
    e = torch.empty((0, h), device="cuda")
    z = torch.empty(0, device="cuda")
    c.block_norm_forward(e, e, v["w_post"], None, v["w_pre"], e, e, z, z)
    c.block_norm_backward(e, e, e, e, v["w_post"], None, v["w_pre"], z, z, e, e, a[0], None, a[2])
    assert not a[0].any() and not a[2].any()


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    t, h = 12, 700
    d = _inputs(t, h, torch.float32, 0, seed=3)
    d["x"][2] = 0; d["y"][2] = 0
    d["x"][5, 3] = math.inf
    d["y"][7, 3] = math.nan
    v = _dev(d)
    n, xo = torch.empty_like(v["x"]), torch.empty_like(v["x"])
    ctx().block_norm_forward(v["x"], v["y"], v["w_post"], None, v["w_pre"], xo, n)
    assert not xo[2].any() and not n[2].any()                       # 0 * eps^-1/2
    rows = [r for r in range(t) if r not in (5, 7)]
    assert bool(torch.isfinite(n[rows]).all()) and bool(torch.isfinite(xo[rows]).all())
    assert bool(xo[7].isnan().all()) and bool(n[7].isnan().all()) and bool(n[5, 3].isnan())


def test_refusals():
    c = ctx()
    x = torch.zeros((4, 64), device="cuda")
    w, g = torch.ones(64, device="cuda"), torch.ones((1, 64), device="cuda")
    r = torch.zeros(4, device="cuda")
    with pytest.raises(edgc.EdgcError):
        c.block_norm_forward(x, None, None, None, None, x, None)                                # neither norm
    with pytest.raises(edgc.EdgcError):
        c.block_norm_forward(x, x, None, None, w, x, x)                                         # y without w_post
    with pytest.raises(edgc.EdgcError):
        c.block_norm_forward(x, x, w, None, w, x, x, eps=-1.0)
    with pytest.raises(edgc.EdgcError):
        c.block_norm_forward(x, x, w, None, w, x, x, scale=math.inf)
    with pytest.raises(ValueError):
        c.block_norm_forward(x, x, w, g, w, x, x)                                               # no rows_per_gate
    with pytest.raises(ValueError):
        c.block_norm_forward(x, x, w, g, w, x, x, rows_per_gate=2)                              # gate of another shape
    with pytest.raises(ValueError):
        c.block_norm_forward(x.t(), x, w, None, w, x, x)
    with pytest.raises(TypeError):
        c.block_norm_forward(x, x.bfloat16(), w, None, w, x, x)
    with pytest.raises(TypeError):
        c.block_norm_forward(x.double(), None, None, None, w.double(), None, x.double())
    big = torch.zeros((1, 16385), device="cuda")
    with pytest.raises(edgc.EdgcError):
        c.block_norm_forward(big, None, None, None, torch.ones(16385, device="cuda"), None, big)
    c.reserve_block_norm(2, 64)
    with pytest.raises(edgc.EdgcError):
        c.block_norm_backward(x, x, x, x, w, None, w, r, r, x, x, w, None, w)                   # more tokens than reserved
    with pytest.raises(edgc.EdgcError):
        c.reserve_block_norm(4, 0)

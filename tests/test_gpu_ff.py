"""The gated feed-forward block, forward and backward, against 64-bit arithmetic."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu

# Every output is a sum over k of products; it is held, element by element, against the sum of the products' absolute values.
# fp32: k terms accumulated in fp32 in some order are off by at most k 2^-24 of that, in the mean by sqrt(k) 2^-24; the operands'
# three planes leave out 2^-22 at most, and what is computed before the last product (A, dG, dU: expf, the activation, a product)
# is off by some 8 units of 2^-23.  128 units of 2^-23 cover k to 20000 in the mean with a wide margin.
# bf16: the intermediate operand and the output are rounded once each: 2^-8 of the terms' sum and 2^-8 of the output; what the
# rounding of an operand does to the other factors of a term (act' of a kept projection is exact) adds nothing.
UNIT = 2.0 ** -23
TOL = {torch.float32: 128 * UNIT, torch.bfloat16: 128 * UNIT + 2 * 2.0 ** -8}

ACTS = ["silu", "gelu", "gelu_tanh"]


def _act64(name, z):
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    s = torch.sigmoid(2 * k * (z + 0.044715 * z ** 3))         # (1 + tanh) / 2, without its cancellation
    return z * s, s + 2 * z * s * (1 - s) * k * (1 + 3 * 0.044715 * z * z)


def _inputs(t, h, f, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std=1.0: (std * torch.randn(*s, generator=g)).to(dtype)
    return dict(x=r(t, h), w_gate=r(f, h, std=h ** -0.5), w_up=r(f, h, std=h ** -0.5), w_down=r(h, f, std=f ** -0.5),
                gate=r(t, f, std=1.5), up=r(t, f), dy=r(t, h, std=1e-2))


def _padded(m, pad, fill=7.0, shift=0):
    """m on the GPU as a view of a buffer whose rows are `pad` elements longer, begun `shift` elements in."""
    if not pad and not shift:
        return m.cuda(), None
    buf = torch.full((m.shape[0] * (m.shape[1] + pad) + shift,), fill, dtype=m.dtype, device="cuda")
    v = buf[shift:].view(m.shape[0], m.shape[1] + pad)[:, :m.shape[1]]
    v.copy_(m)
    return v, buf


def _close(got, want, size, what):
    got, tol = got.cpu(), TOL[got.dtype]
    err = (got.double() - want).abs() / size.clamp_min(1e-30)
    assert bool((err <= tol).all()), (what, float(err.max()), tol)


def _forward_check(d, act, y, gate=None, up=None):
    q = {k: v.double() for k, v in d.items()}
    G, U = q["x"] @ q["w_gate"].t(), q["x"] @ q["w_up"].t()
    Gs, Us = q["x"].abs() @ q["w_gate"].t().abs(), q["x"].abs() @ q["w_up"].t().abs()
    a, da = _act64(act, G)
    A = a * U
    # A is off by what its two factors are off by
    As = a.abs() * Us + da.abs().clamp_min(0.1) * Gs * U.abs()
    k = 1.0 if y.dtype == torch.float32 else UNIT * 128 / (128 * UNIT + 2.0 ** -8)
    size = A.abs() @ q["w_down"].t().abs() + k * (As @ q["w_down"].t().abs())
    _close(y, A @ q["w_down"].t(), size, "y")
    if gate is not None:
        _close(gate, G, Gs, "gate")
        _close(up, U, Us, "up")


def _backward_check(d, act, out, base=None):
    q = {k: v.double() for k, v in d.items()}
    a, da = _act64(act, q["gate"])
    dA, dAs = q["dy"] @ q["w_down"], q["dy"].abs() @ q["w_down"].abs()
    dG, dU, A = dA * q["up"] * da, dA * a, a * q["up"]
    dGs, dUs = dAs * q["up"].abs() * da.abs().clamp_min(0.01), dAs * a.abs().clamp_min(0.01)
    if base is None:
        base = {k: torch.zeros_like(q[k[1:]]) for k in out}
    add = lambda k, v, s: _close(out[k], base[k].double() + v, base[k].double().abs() + s, k)
    add("dx", dG @ q["w_gate"] + dU @ q["w_up"], dGs @ q["w_gate"].abs() + dUs @ q["w_up"].abs())
    add("dw_gate", dG.t() @ q["x"], dGs.t() @ q["x"].abs())
    add("dw_up", dU.t() @ q["x"], dUs.t() @ q["x"].abs())
    add("dw_down", q["dy"].t() @ A, q["dy"].abs().t() @ A.abs())


# tokens, hidden, ff: one and few tokens, tiles that end inside, sizes that no unit divides, several tiles either way, long k
SIZES = [(1, 64, 128), (1, 1000, 2730), (1, 1, 1), (2, 3, 5), (5, 640, 1536), (16, 512, 2048), (17, 129, 65), (31, 257, 511),
         (33, 64, 64), (64, 256, 256), (100, 77, 300), (130, 320, 200), (255, 192, 1024), (257, 513, 259), (300, 1024, 640),
         (1025, 128, 384), (64, 4096, 128), (48, 128, 4096), (700, 2048, 1100)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h,f", SIZES)
@pytest.mark.parametrize("keep", [False, True])
def test_forward(t, h, f, dtype, keep):
    act = ACTS[(t + h + f) % 3]
    d = _inputs(t, h, f, dtype)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(dtype, t, h, f)
    y = torch.full((t, h), 7.0, dtype=dtype, device="cuda")
    g, u = (torch.full((t, f), 7.0, dtype=dtype, device="cuda") if keep else None for _ in range(2))
    c.ff_forward(edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], act), v["x"], y, g, u)
    _forward_check(d, act, y, g, u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h,f", SIZES)
def test_backward(t, h, f, dtype):
    act = ACTS[(t + h + f) % 3]
    d = _inputs(t, h, f, dtype, seed=1)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    out = {"d" + k: torch.full_like(v[k], 7.0) for k in ("x", "w_gate", "w_up", "w_down")}
    c.ff_backward(edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], act), v["x"], v["gate"], v["up"], v["dy"], out["dx"],
                  out["dw_gate"], out["dw_up"], out["dw_down"])
    _backward_check(d, act, out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pads", [dict(x=8, w_gate=16), dict(x=3, w_gate=1, w_up=5, w_down=7, dy=1, gate=2, up=2, y=3),
                                  dict(w_up=64), dict(shift=1), dict(shift=4, w_down=64, x=64)], ids=str)
@pytest.mark.parametrize("t,h,f", [(70, 192, 320), (1, 128, 256), (300, 130, 270)])
def test_strides_and_alignment(t, h, f, dtype, pads):
    """Rows further apart than they are long, of lengths that no unit divides, begun off any boundary; what lies between the rows
    is not touched."""
    d = _inputs(t, h, f, dtype, seed=2)
    s = pads.get("shift", 0)
    v, bufs = {}, {}
    for k, a in d.items():
        v[k], bufs[k] = _padded(a, pads.get(k, 0), shift=s)
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    out, ob = {}, {}
    for k in ("x", "w_gate", "w_up", "w_down"):
        out["d" + k], ob["d" + k] = _padded(torch.zeros_like(d[k]), pads.get(k, 0), shift=s)
    out["y"], ob["y"] = _padded(torch.zeros_like(d["x"]), pads.get("y", 0), shift=s)
    out["gate"], ob["gate"] = _padded(torch.zeros_like(d["gate"]), pads.get("gate", 0), shift=s)
    out["up"], ob["up"] = _padded(torch.zeros_like(d["up"]), pads.get("up", 0), shift=s)
    w = edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], "gelu")
    c.ff_forward(w, v["x"], out["y"], out["gate"], out["up"])
    _forward_check(d, "gelu", out["y"], out["gate"], out["up"])
    c.ff_backward(w, v["x"], v["gate"], v["up"], v["dy"], out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"])
    _backward_check(d, "gelu", {k: out[k] for k in ("dx", "dw_gate", "dw_up", "dw_down")})
    for k, b in list(ob.items()) + list(bufs.items()):
        if b is None:
            continue
        m = out[k] if k in ob and b is ob[k] else v[k]
        mask = torch.ones_like(b, dtype=torch.bool)
        mask[s:].view(m.shape[0], -1)[:, :m.shape[1]] = False
        assert bool((b[mask] == 7).all()), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_accumulation_over_micro_batches(dtype):
    t, h, f = 90, 256, 300
    d, e = _inputs(t, h, f, dtype, seed=3), _inputs(t, h, f, dtype, seed=4)
    e.update({k: d[k] for k in ("w_gate", "w_up", "w_down")})
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    w = edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"])
    out = {"d" + k: torch.full_like(v[k], 7.0) for k in ("x", "w_gate", "w_up", "w_down")}
    c.ff_backward(w, v["x"], v["gate"], v["up"], v["dy"], out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"])
    base = {k: o.cpu().clone() for k, o in out.items()}
    base["dx"] = torch.zeros_like(base["dx"])               # dx is of the micro-batch at hand
    v = {k: a.cuda() for k, a in e.items()}
    c.ff_backward(w, v["x"], v["gate"], v["up"], v["dy"], out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"], accumulate=True)
    _backward_check(e, "silu", out, base)
    none = {k: v[k][:0] for k in ("x", "gate", "up", "dy")}
    before = out["dw_up"].clone()
    c.ff_backward(w, none["x"], none["gate"], none["up"], none["dy"], out["dx"][:0], out["dw_gate"], out["dw_up"], out["dw_down"],
                  accumulate=True)
    assert torch.equal(before, out["dw_up"])
    c.ff_forward(w, none["x"], none["x"].clone())
    c.ff_backward(w, none["x"], none["gate"], none["up"], none["dy"], out["dx"][:0], out["dw_gate"], out["dw_up"], out["dw_down"])
    assert not out["dw_gate"].any() and not out["dw_up"].any() and not out["dw_down"].any()


@pytest.mark.parametrize("act", ACTS)
def test_gradients_are_the_differences_of_the_forward_pass(act):
    """fp32 gradients through forward and backward along random directions against central differences in 64 bits."""
    t, h, f = 20, 96, 160
    d = _inputs(t, h, f, torch.float32, seed=5)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(torch.float32, t, h, f, backward=True)
    w = edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], act)
    y = torch.empty_like(v["x"])
    c.ff_forward(w, v["x"], y, v["gate"], v["up"])
    out = {k: torch.empty_like(v[k]) for k in ("x", "w_gate", "w_up", "w_down")}
    c.ff_backward(w, v["x"], v["gate"], v["up"], v["dy"], out["x"], out["w_gate"], out["w_up"], out["w_down"])

    def loss(q):
        q = {k: a.double() for k, a in q.items()}
        return float((((_act64(act, q["x"] @ q["w_gate"].t())[0] * (q["x"] @ q["w_up"].t())) @ q["w_down"].t()) * q["dy"]).sum())
    g = torch.Generator().manual_seed(6)
    for k, grad in out.items():
        e = torch.randn(d[k].shape, generator=g, dtype=torch.float64)
        step = 1e-5
        hi, lo = dict(d), dict(d)
        hi[k], lo[k] = d[k].double() + step * e, d[k].double() - step * e
        diff = (loss(hi) - loss(lo)) / (2 * step)
        size = float((grad.cpu().double() * e).abs().sum())
        # fp32 sums against the sum of the terms, and the differences' step^2 and 64-bit cancellation
        assert abs(float((grad.cpu().double() * e).sum()) - diff) <= (128 * UNIT + 1e-6) * size, k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ACTS)
def test_projections_of_any_size(dtype, act):
    """Kept projections far outside the activation's bend: nothing overflows on the way to a finite value."""
    t, h, f = 40, 64, 128
    d = _inputs(t, h, f, dtype, seed=7)
    d["gate"] = (d["gate"].float() * 10.0 ** torch.linspace(-6, 6, t)[:, None]).to(dtype)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    out = {"d" + k: torch.full_like(v[k], 7.0) for k in ("x", "w_gate", "w_up", "w_down")}
    c.ff_backward(edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], act), v["x"], v["gate"], v["up"], v["dy"], out["dx"],
                  out["dw_gate"], out["dw_up"], out["dw_down"])
    assert all(bool(torch.isfinite(o).all()) for o in out.values())
    _backward_check(d, act, out)


def test_what_is_not_finite_stays_in_its_row():
    t, h, f = 40, 256, 320
    for dtype in (torch.float32, torch.bfloat16):
        d = _inputs(t, h, f, dtype, seed=8)
        d["x"][3, 5], d["x"][9, 0] = math.inf, math.nan
        v = {k: a.cuda() for k, a in d.items()}
        c = ctx()
        c.reserve_ff(dtype, t, h, f)
        y = torch.empty_like(v["x"])
        c.ff_forward(edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"]), v["x"], y)
        rows = [r for r in range(t) if r not in (3, 9)]
        assert bool(torch.isfinite(y[rows]).all()) and not bool(torch.isfinite(y[3]).any()) and bool(y[9].isnan().all())


def test_the_same_bits_every_time_and_on_another_stream():
    t, h, f = 200, 512, 768
    d = _inputs(t, h, f, torch.bfloat16, seed=9)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(torch.bfloat16, t, h, f, backward=True)
    w = edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"])

    def go():
        out = [torch.full_like(v[k], 7.0) for k in ("x", "x", "w_gate", "w_up", "w_down")]
        c.ff_forward(w, v["x"], out[0])
        c.ff_backward(w, v["x"], v["gate"], v["up"], v["dy"], *out[1:])
        return out
    first = go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = go()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_refusals():
    c = ctx()
    x = torch.zeros((4, 64), device="cuda")
    wg, wd = torch.zeros((128, 64), device="cuda"), torch.zeros((64, 128), device="cuda")
    k = torch.zeros((4, 128), device="cuda")
    c.reserve_ff(torch.float32, 4, 64, 128)
    w = edgc.FeedForward(wg, wg, wd)
    with pytest.raises(ValueError):
        edgc.FeedForward(wg, wg, wd, "tanh")
    with pytest.raises(ValueError):
        edgc.FeedForward(wg, wg, wg)
    with pytest.raises(ValueError):
        edgc.FeedForward(wd.t(), wd.t(), wg.t())                    # rows that are not contiguous
    with pytest.raises(TypeError):
        edgc.FeedForward(wg, wg.bfloat16(), wd)
    with pytest.raises(TypeError):
        edgc.FeedForward(wg.half(), wg.half(), wd.half())
    with pytest.raises(TypeError):
        c.reserve_ff(torch.float16, 4, 64, 128)
    with pytest.raises(ValueError):
        c.ff_forward(w, x, x[:, :32])
    with pytest.raises(TypeError):
        c.ff_forward(w, x.bfloat16(), x)
    with pytest.raises(edgc.EdgcError):
        c.ff_forward(w, x, torch.empty_like(x), k, None)            # one of the two projections
    big = torch.zeros((1000, 64), device="cuda")
    with pytest.raises(edgc.EdgcError):
        c.ff_forward(w, big, torch.empty_like(big))                 # over the reservation
    c.reserve_ff(torch.float32, 4, 64, 128)
    with pytest.raises(edgc.EdgcError):
        c.reserve_ff(torch.float32, 4, 0, 128)

"""The feed-forward block's products, each way that they are split over tiles, waves and workers, held to bounds that a lost share
of a sum does not pass: element by element against 64 bits, relative to the root of the sum of the terms' squares."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx
from test_gpu_ff import ACTS, SIZES, _act64

pytestmark = pytest.mark.gpu

# An output is a sum of k products a b, of which a (A, dG, dU) may have been rounded to bf16: by at most R = 2^-8 of itself, in a way
# that has nothing to do with b.  The errors' sum is then of the size R / 2 sqrt(V), V = sum (a b)^2; 4 R sqrt(V) is eight of its
# deviations, and for up to 16 terms the largest that it can be at all.  The output's own rounding: R of itself.
# fp32 arithmetic: n roundings of partial sums of the size of sqrt(V), n below 1700 for the k here, 16 to 20 units of 2^-23 in
# the mean and four times that at the most; 128 cover them and the activations'.  What precedes the last product is off by as much of its
# own root of V, which is what the sums W below carry.
R = 2.0 ** -8
UNIT = 2.0 ** -23
N = 128 * UNIT


def _inputs(t, h, f, dtype, seed, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)

    def r(*s, std=1.0):
        m = torch.empty(s, device=device, dtype=dtype)
        for part in m.split(max(1, (1 << 25) // s[1])):
            part.copy_(torch.randn(part.shape, generator=g, device=device).mul_(std))
        return m
    return dict(x=r(t, h), w_gate=r(f, h, std=h ** -0.5), w_up=r(f, h, std=h ** -0.5), w_down=r(h, f, std=f ** -0.5),
                gate=r(t, f, std=1.5), up=r(t, f), dy=r(t, h, std=1e-2))


def _check(what, got, want, rounded, before):
    """got against want; `rounded`: V of what was rounded to bf16 before the product, `before`: W, of fp32's own errors."""
    bf16 = got.dtype == torch.bfloat16
    tol = (R if bf16 else 2 * UNIT) * want.abs() + N * before.sqrt() + 1e-37
    if bf16 and rounded is not None:
        tol = tol + 4 * R * rounded.sqrt()
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (what, float((err / tol).max()), int((err > tol).sum()), err.numel())


def _forward_check(d, act, y, gate=None, up=None):
    q = {k: d[k].double() for k in ("x", "w_gate", "w_up", "w_down")}
    G, U = q["x"] @ q["w_gate"].t(), q["x"] @ q["w_up"].t()
    VG, VU = q["x"].square() @ q["w_gate"].square().t(), q["x"].square() @ q["w_up"].square().t()
    if gate is not None:
        _check("gate", gate, G, None, VG)
        _check("up", up, U, None, VU)
    a, da = _act64(act, G)
    A = a * U
    WA = A.square() + a.square() * VU + (da.abs().clamp_min(0.25) * U).square() * VG
    wd2 = q["w_down"].square().t()
    _check("y", y, A @ q["w_down"].t(), A.square() @ wd2, WA @ wd2)


def _backward_check(d, act, out, base=None):
    q = {k: v.double() for k, v in d.items()}
    a, da = _act64(act, q["gate"])
    dA, VA = q["dy"] @ q["w_down"], q["dy"].square() @ q["w_down"].square()
    A, dG, dU = a * q["up"], dA * q["up"] * da, dA * a
    # the derivative passes through zero and is off by some units of 1 + |z| there
    WA, WG, WU = A.square(), VA * (q["up"] * da.abs().clamp_min(0.25)).square(), VA * a.square()
    s = {k: q[k].square() for k in ("x", "w_gate", "w_up", "dy")}

    def hold(k, want, rounded, before):
        if base is not None and k != "dx":
            want, before = want + base[k].double(), before + base[k].double().square()
        _check(k, out[k], want, rounded, before)
    hold("dx", dG @ q["w_gate"] + dU @ q["w_up"], dG.square() @ s["w_gate"] + dU.square() @ s["w_up"], WG @ s["w_gate"] + WU @ s["w_up"])
    hold("dw_gate", dG.t() @ q["x"], dG.square().t() @ s["x"], WG.t() @ s["x"])
    hold("dw_up", dU.t() @ q["x"], dU.square().t() @ s["x"], WU.t() @ s["x"])
    hold("dw_down", q["dy"].t() @ A, s["dy"].t() @ A.square(), s["dy"].t() @ WA)


def _forward(t, h, f, dtype, keep, seed=0):
    act = ACTS[(t + h + f) % 3]
    d = _inputs(t, h, f, dtype, seed)
    c = ctx()
    c.reserve_ff(dtype, t, h, f)
    y = torch.full((t, h), 7.0, dtype=dtype, device="cuda")
    g, u = (torch.full((t, f), 7.0, dtype=dtype, device="cuda") if keep else None for _ in range(2))
    c.ff_forward(edgc.FeedForward(d["w_gate"], d["w_up"], d["w_down"], act), d["x"], y, g, u)
    _forward_check(d, act, y, g, u)


def _backward(t, h, f, dtype, accumulate=False, seed=1):
    act = ACTS[(t + h + f) % 3]
    d = _inputs(t, h, f, dtype, seed)
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    out = {"d" + k: torch.full_like(d[k], 7.0) for k in ("x", "w_gate", "w_up", "w_down")}
    if accumulate:
        g = torch.Generator(device="cuda").manual_seed(5)
        for k in ("dw_gate", "dw_up", "dw_down"):
            out[k].copy_(torch.randn(out[k].shape, generator=g, device="cuda").mul_(0.1))
    base = {k: v.clone() for k, v in out.items()} if accumulate else None
    c.ff_backward(edgc.FeedForward(d["w_gate"], d["w_up"], d["w_down"], act), d["x"], d["gate"], d["up"], d["dy"], out["dx"],
                  out["dw_gate"], out["dw_up"], out["dw_down"], accumulate=accumulate)
    _backward_check(d, act, out, base)


DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t,h,f", SIZES)
def test_forward(t, h, f, dtype):
    _forward(t, h, f, dtype, keep=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t,h,f", SIZES)
def test_backward(t, h, f, dtype):
    _backward(t, h, f, dtype)


# On 256 compute units: whole rounds of 256 x 256 tiles and a shared rest in every product of both passes, k of 10 steps and more, ends
# inside tiles, operands as they stand and copied; of 128 x 128 tiles the same in the gradients of the projections.
LARGE = [(4200, 4232, 640), (4200, 640, 4240), (640, 2600, 2600), (640, 2624, 2688), (3200, 448, 2944)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t,h,f", LARGE)
def test_forward_of_whole_rounds_and_a_shared_rest(t, h, f, dtype):
    _forward(t, h, f, dtype, keep=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("t,h,f", LARGE)
def test_backward_of_whole_rounds_and_a_shared_rest(t, h, f, dtype, accumulate):
    _backward(t, h, f, dtype, accumulate)


# Few tokens: 16 waves a block; long loops of either buffer; k shared by two and four blocks, in the projections and after them, with a
# step that ends inside; one, two and (fp32) four groups of tokens.
FEW = [(1, 4096, 16384), (20, 4096, 16384), (7, 1000, 8197), (1, 1000, 4099), (30, 8192, 1000), (16, 8200, 1003), (32, 2048, 4100), (50, 2048, 4100),
       (64, 1000, 8200)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("t,h,f", FEW)
def test_few_tokens_of_long_rows(t, h, f, dtype, keep):
    _forward(t, h, f, dtype, keep)


def test_few_tokens_of_long_rows_again_and_again():
    """Blocks that share k leave their places as they found them: the same bits in calls of one shape after those of another."""
    c = ctx()
    shapes = [(7, 1000, 8197), (30, 8192, 1000), (1, 1000, 4099)]
    for dtype in DTYPES:
        c.reserve_ff(dtype, 30, 8192, 8197)
        runs = []
        for t, h, f in shapes:
            d = _inputs(t, h, f, dtype, 3)
            runs.append((edgc.FeedForward(d["w_gate"], d["w_up"], d["w_down"]), d["x"]))
        first = None
        for _ in range(4):
            ys = [torch.full_like(x, 7.0) for _, x in runs]
            for (w, x), y in zip(runs, ys):
                c.ff_forward(w, x, y)
            first = first or ys
            assert all(torch.equal(a, b) for a, b in zip(first, ys))

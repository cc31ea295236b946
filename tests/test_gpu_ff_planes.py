"""fp32 products made of planes, each of the five kinds of product by itself, with sums so short that every product of planes counts."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

# Operands between 1 and 2 (or 32 and 64) with all 24 bits, K = 8 or 16 terms of one sign that are not zero.  An operand is p0 + p1 + p2, cut to
# eight bits each: p1 < 2^-7 p0, p2 < 2^-15 p0.  p1 q2 + p2 q1 + p2 q2 are left out: below 2^-21 of the product.  Each of at most K sums
# of the leading products is off by one unit, 2^-23, of the result, those of the others by 2^-7 of that, an operand that is itself
# computed by up to two units: (K + 3) 2^-23 + 2^-21, and one unit for the rounding.
UNIT = 2.0 ** -23


def tolerance(k):
    return (k + 8) * UNIT


def _full(g, *s, device):
    """In [1, 2), no bit of the 24 left alone."""
    return (1 + torch.randint(0, 1 << 23, s, generator=g, device=device).double() * 2.0 ** -23).float()


# What is handed in, and the products that are seen, as (name of the output, left operand, right operand): left right^T
def projections(t, h, f, device="cuda"):
    g = torch.Generator(device=device).manual_seed(1)
    x, wg, wu = torch.zeros(t, h, device=device), torch.zeros(f, h, device=device), torch.zeros(f, h, device=device)
    for m in (x, wg, wu):
        m[:, :8] = _full(g, m.shape[0], 8, device=device)
    return dict(x=x, w_gate=wg, w_up=wu, w_down=torch.zeros(h, f, device=device)), [("gate", x, wg), ("up", x, wu)], 8


def down(t, h, f, device="cuda"):
    """x picks rows of the weights, and an activation that is the identity leaves A = w_gate's."""
    g = torch.Generator(device=device).manual_seed(2)
    at = torch.arange(t, device=device) % h
    x = torch.zeros(t, h, device=device)
    x[torch.arange(t, device=device), at] = 1.0
    wg, wd = torch.zeros(f, h, device=device), torch.zeros(h, f, device=device)
    wg[:8], wd[:, :8] = 32 * _full(g, 8, h, device=device), _full(g, h, 8, device=device)
    A = wg.t()[at]
    return dict(x=x, w_gate=wg, w_up=torch.ones(f, h, device=device), w_down=wd), [("y", A, wd)], 8


def gradient_of_the_projections(t, h, f, device="cuda"):
    """x is the identity, so that dw_gate is dG, and dG = dA."""
    g = torch.Generator(device=device).manual_seed(3)
    dy, wd = torch.zeros(t, h, device=device), torch.zeros(h, f, device=device)
    dy[:, :8], wd[:8] = _full(g, t, 8, device=device), _full(g, 8, f, device=device)
    d = dict(x=torch.eye(t, h, device=device), w_gate=torch.zeros(f, h, device=device), w_up=torch.zeros(f, h, device=device), w_down=wd,
             gate=torch.full((t, f), 40.0, device=device), up=torch.ones(t, f, device=device), dy=dy)
    return d, [("dw_gate", wd.t().contiguous(), torch.nn.functional.pad(dy, (0, 0, 0, h - t)))], 8


def dx(t, h, f, device="cuda"):
    """w_down picks columns of dy: dG = dA up, dU = dA gate."""
    g = torch.Generator(device=device).manual_seed(4)
    dy, gate, up = _full(g, t, h, device=device), 32 * _full(g, t, f, device=device), 32 * _full(g, t, f, device=device)
    wg, wu = torch.zeros(f, h, device=device), torch.zeros(f, h, device=device)
    wg[:8], wu[:8] = _full(g, 8, h, device=device), _full(g, 8, h, device=device)
    d = dict(x=torch.zeros(t, h, device=device), w_gate=wg, w_up=wu, w_down=torch.eye(h, f, device=device), gate=gate, up=up, dy=dy)
    dA = dy[:, :f]
    return d, [("dx", torch.cat([dA * up, dA * gate], 1), torch.cat([wg, wu], 0).t())], 16


def weights(t, h, f, device="cuda"):
    g = torch.Generator(device=device).manual_seed(5)
    dy, x = _full(g, t, h, device=device), _full(g, t, h, device=device)
    gate, up = 32 * _full(g, t, f, device=device), _full(g, t, f, device=device)
    wd, at = torch.zeros(h, f, device=device), torch.arange(f, device=device)
    wd[at % h, at] = 1.0
    d = dict(x=x, w_gate=torch.zeros(f, h, device=device), w_up=torch.zeros(f, h, device=device), w_down=wd, gate=gate, up=up, dy=dy)
    dA = dy[:, at % h]
    return d, [("dw_gate", (dA * up).t(), x.t()), ("dw_up", (dA * gate).t(), x.t()), ("dw_down", dy.t(), (gate * up).t())], t


# one tile that ends inside, several of the smaller shape, and enough for the larger one
CASES = [(projections, 200, 8, 300), (projections, 40, 8, 300), (projections, 3000, 8, 2600), (down, 200, 150, 8), (down, 33, 150, 8),
         (down, 4000, 4000, 8), (gradient_of_the_projections, 70, 100, 300), (gradient_of_the_projections, 2000, 2000, 2600), (dx, 200, 300, 8),
         (dx, 4000, 4000, 8), (weights, 8, 200, 300), (weights, 8, 4000, 4000)]
NAMES = [f"{c[0].__name__}-{c[1]}x{c[2]}x{c[3]}" for c in CASES]


@pytest.mark.gpu
@pytest.mark.parametrize("make,t,h,f", CASES, ids=NAMES)
def test_short_sums_of_whole_operands(make, t, h, f):
    d, seen, k = make(t, h, f)
    w = edgc.FeedForward(d["w_gate"], d["w_up"], d["w_down"], "silu")
    c = ctx()
    c.reserve_ff(torch.float32, t, h, f, backward="dy" in d)
    out = {}
    if "dy" in d:
        out = {"d" + n: torch.full_like(d[n], 7.0) for n in ("x", "w_gate", "w_up", "w_down")}
        c.ff_backward(w, d["x"], d["gate"], d["up"], d["dy"], out["dx"], out["dw_gate"], out["dw_up"], out["dw_down"])
    else:
        out = {"y": torch.full_like(d["x"], 7.0), "gate": torch.full((t, f), 7.0, device="cuda"), "up": torch.full((t, f), 7.0, device="cuda")}
        c.ff_forward(w, d["x"], out["y"], out["gate"], out["up"])
    for name, a, b in seen:
        want = a.double() @ b.double().t()
        err = (out[name].double() - want).abs()
        assert bool((err <= tolerance(k) * want).all()), (name, float((err / want.clamp_min(1e-30)).max()) / UNIT)


def _planes(x):
    """As the kernels cut them: three times eight bits."""
    out = []
    for _ in range(3):
        p = (x.contiguous().view(torch.int32) & -65536).view(torch.float32)
        out.append(p)
        x = x - p
    assert not x.any()
    return out


@pytest.mark.parametrize("make,t,h,f", [(projections, 64, 8, 96), (down, 64, 48, 8), (gradient_of_the_projections, 40, 64, 96), (dx, 64, 96, 8),
                                        (weights, 8, 64, 96)], ids=lambda v: getattr(v, "__name__", v))
def test_the_bound_tells_six_products_from_five(make, t, h, f):
    """On the CPU: the six products of planes meet the bound with room, and any five of them do not."""
    _, seen, k = make(t, h, f, device="cpu")
    for _, a, b in seen:
        want = a.double() @ b.double().t()
        pa, pb = _planes(a), _planes(b)
        six = {(i, j): pa[i].double() @ pb[j].double().t() for i in range(3) for j in range(3) if i + j <= 2}
        assert float(((sum(six.values()) - want).abs() / want.clamp_min(1e-30)).max()) <= 4 * UNIT
        for lost in six:
            worst = float(((sum(v for s, v in six.items() if s != lost) - want).abs() / want.clamp_min(1e-30)).max())
            assert worst > 2 * tolerance(k), (lost, worst / UNIT)

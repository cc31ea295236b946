"""The activations of the feed-forward block and their derivatives over the whole line, element by element."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu

# Weights of ones and zeros make y = act(z) and dx = act'(z): every sum has one term that is not zero, and fp32 products are exact.
# act(z) = z s(z), 0 <= s <= 1: s is made of a power of two, a reciprocal and up to ten multiply-adds, each off by 2^-24 to 2^-23 of
# its result, and its argument, off by 3 2^-24 of itself, moves s by u s (1 - s) < 0.3 times that: 2^-21 of |z| covers both.
# act'(z) = s + z s (1 - s) .. (or a density times z, below 1/4): 1 - s is off by 2^-24 where s is near 1, times |z|, and the rest as
# above, its factors' errors added up: 2^-20 (1 + |z|).
FORWARD, BACKWARD = 2.0 ** -21, 2.0 ** -20


def _act64(name, z):
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * torch.sigmoid(-z))
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    k, u = math.sqrt(2 / math.pi), 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    s = torch.sigmoid(u)
    return z * s, s + 2 * z * s * torch.sigmoid(-u) * k * (1 + 3 * 0.044715 * z * z)


# tokens that go to the kernel of few tokens, and to the tiles
@pytest.mark.parametrize("tokens", [40, 520])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activation_and_derivative(act, tokens):
    h = 64
    z = torch.cat([torch.linspace(-30, 30, tokens * (h - 1) - 8), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-8, -1e-8, 300.0, -300.0])])
    z = z.view(tokens, h - 1)
    one = torch.ones(tokens, 1)
    x = torch.cat([z, one], 1).cuda()
    f = h - 1
    w_gate = torch.eye(f, h).cuda()                     # G = z
    w_up = torch.zeros(f, h).cuda()
    w_up[:, h - 1] = 1.0                                # U = 1
    w_down = torch.eye(h, f).cuda()                     # y = A, and a zero
    w = edgc.FeedForward(w_gate, w_up, w_down, act)
    c = ctx()
    c.reserve_ff(torch.float32, tokens, h, f, backward=True)
    y, gate, up = torch.empty_like(x), torch.empty(tokens, f, device="cuda"), torch.empty(tokens, f, device="cuda")
    c.ff_forward(w, x, y, gate, up)
    assert torch.equal(gate.cpu(), z) and bool((up == 1).all())
    a, da = _act64(act, z.double())
    err = (y[:, :f].cpu().double() - a).abs()
    assert bool((err <= FORWARD * z.double().abs() + 1e-37).all()), float((err / z.double().abs().clamp_min(1e-37)).max())
    # dA = 1 where y is A; dx = dG in the first columns
    dy = torch.cat([torch.ones(tokens, f), torch.zeros(tokens, 1)], 1).cuda()
    dx, dw = torch.empty_like(x), [torch.empty_like(m) for m in (w_gate, w_up, w_down)]
    c.ff_backward(w, x, gate, up, dy, dx, *dw)
    err = (dx[:, :f].cpu().double() - da).abs()
    assert bool((err <= BACKWARD * (1 + z.double().abs())).all()), float((err / (1 + z.double().abs())).max())

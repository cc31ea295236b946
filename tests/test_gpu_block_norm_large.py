"""The norms' backward pass with a gate where element offsets pass 32 bits: rows of dy and dx from all over, columns of every sum."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from test_gpu_block_large import UNIT, _randn, _room

pytestmark = pytest.mark.gpu


def test_backward_with_gates_beyond_32_bit_offsets():
    _room(96)
    t, h, per, scale = 140001, 16384, 5003, 0.5                 # 2.3e9 elements, 28 rows of the gate, the last one short
    groups = -(-t // per)
    xo, y, dn, dxo = _randn(t, h, 1), _randn(t, h, 2, 3.0), _randn(t, h, 3, 1e-2), _randn(t, h, 4, 1e-2)
    wp, wn, gate = _randn(1, h, 5)[0], _randn(1, h, 6)[0], _randn(groups, h, 7)
    rstd = lambda m: torch.cat([torch.rsqrt(p.float().square().mean(1) + 1e-6) for p in m.split(4096)])
    r1, r2 = rstd(y), rstd(xo)
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.reserve_block_norm(t, h)
    dx, dy, dgate = torch.full_like(xo, 7.0), torch.full_like(xo, 7.0), torch.full_like(gate, 7.0)
    dwp, dwn = torch.full_like(wp, 7.0), torch.full_like(wn, 7.0)
    ctx.block_norm_backward(dxo, dn, xo, y, wp, gate, wn, r1, r2, dx, dy, dwp, dgate, dwn, scale=scale, rows_per_gate=per)

    def rows(i):
        """D, u, xh, yh of some rows in 64 bits, and the size of the terms that D is made of."""
        xh, yh = xo[i].double() * r2[i].double()[:, None], y[i].double() * r1[i].double()[:, None]
        u, r = dn[i].double() * wn.double(), r2[i].double()[:, None]
        D = dxo[i].double() + r * (u - xh * (u * xh).mean(1, keepdim=True))
        size = dxo[i].double().abs() + r * (u.abs() + xh.abs() * (u * xh).abs().mean(1, keepdim=True))
        return D, xh, yh, size
    # 100 units of 2^-23 of the terms' sizes and one rounding to bf16
    tol = 100 * UNIT
    i = torch.tensor([0, 1, per - 1, per, 65535, 131071, 131072, 27 * per, t - 2, t - 1], device="cuda")
    D, xh, yh, size = rows(i)
    assert bool(((dx[i].double() - D).abs() <= tol * size + 2.0 ** -8 * D.abs()).all())
    c = scale * gate[i // per].double() * wp.double()
    r = r1[i].double()[:, None]
    want = r * (c * D - yh * (c * D * yh).mean(1, keepdim=True))
    big = r * (c.abs() * size + yh.abs() * (c * D * yh).abs().mean(1, keepdim=True))
    assert bool(((dy[i].double() - want).abs() <= tol * big + 2.0 ** -8 * want.abs()).all())
    cols = torch.tensor([0, 7, 8, 8191, 8192, h - 1], device="cuda")
    zero = lambda *s: torch.zeros(*s, len(cols), device="cuda", dtype=torch.float64)
    S, Sa, pre, pre_a = zero(groups), zero(groups), zero(), zero()
    for part in torch.arange(t, device="cuda").split(2048):
        D, xh, yh, size = (m[:, cols] for m in rows(part))
        S.index_add_(0, part // per, D * yh)
        Sa.index_add_(0, part // per, size * yh.abs())
        pre += (dn[part][:, cols].double() * xh).sum(0)
        pre_a += (dn[part][:, cols].double() * xh).abs().sum(0)
    # fp32 sums of 137 rows by a group and of 128 groups by a thread: 300 units with the terms' own
    tol, wp64, g64 = 300 * UNIT, wp[cols].double(), gate[:, cols].double()

    def hold(got, want, size):
        assert bool(((got.double() - want).abs() <= tol * size + 2.0 ** -8 * want.abs()).all())
    hold(dwn[cols], pre, pre_a)
    hold(dgate[:, cols], scale * wp64 * S, scale * wp64.abs() * Sa)
    hold(dwp[cols], scale * (g64 * S).sum(0), scale * (g64.abs() * Sa).sum(0))
    ctx.close()
    torch.cuda.empty_cache()

"""The gate's gradient where rows of the gate and groups of tokens do not fall together, against 64-bit sums."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -23
# of the sum of the terms' absolute values: fp32 sums of at most 2^13 terms in a fixed order, each term off by some tens of units of
# its factors' sizes; one rounding to bf16 is at most 2^-8 of the result
TOL = {torch.float32: 100 * UNIT, torch.bfloat16: 100 * UNIT + 2.0 ** -8}


def _backward(t, h, dtype, rows_per_gate, groups, seed=0, scale=0.7):
    """Inputs, and the gradients of y alone (no norm after it): dy, dw_post, dgate."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std=1.0: (std * torch.randn(*s, generator=g)).to(dtype)
    y, d, w, gate = r(t, h, std=3.0), r(t, h, std=1e-2), r(h) + 1, r(groups, h)
    rstd = (1 / torch.sqrt((y.double() ** 2).mean(1) + 1e-6)).float()
    out = {"dx": torch.empty_like(y), "dy": torch.empty_like(y), "dw": torch.empty_like(w), "dgate": torch.full_like(gate, 7.0)}
    out = {k: v.cuda() for k, v in out.items()}
    c = ctx()
    c.reserve_block_norm(t, h)
    c.block_norm_backward(d.cuda(), None, None, y.cuda(), w.cuda(), gate.cuda(), None, rstd.cuda(), None, out["dx"], out["dy"], out["dw"],
                          out["dgate"], None, scale=scale, rows_per_gate=rows_per_gate)
    return (y, d, w, gate, rstd), out


def _check(ins, out, rows, scale=0.7):
    y, d, w, gate, rstd = (v.double() for v in ins)
    t, h = y.shape
    per = d * y * rstd[:, None]
    row = torch.arange(t) // rows
    zero = torch.zeros_like(gate)
    S, Sa = zero.index_add(0, row, per), zero.index_add(0, row, per.abs())
    tol = TOL[out["dgate"].dtype]
    got = out["dgate"].cpu().double()
    assert bool(((got - scale * w * S).abs() <= tol * (scale * w.abs() * Sa) + 1e-30).all())
    want, size = scale * (gate * S).sum(0), scale * (gate.abs() * Sa).sum(0)
    assert bool(((out["dw"].cpu().double() - want).abs() <= tol * size).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [2 ** 64 - 1, 2 ** 64 - 2500, 2 ** 63, 2 ** 32, 2500])
@pytest.mark.parametrize("t,h", [(2500, 96), (2500, 1100), (2, 8)])
def test_one_gate_for_everything_by_a_length_beyond_all_tokens(t, h, rows, dtype):
    ins, out = _backward(t, h, dtype, rows, 1)
    _check(ins, out, t)


# rows of the gate of two and three tokens and groups of as many and more: every group but the last may begin one that goes on
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h,rows", [(2500, 96, 2), (2500, 96, 3), (5000, 96, 3), (5000, 96, 4), (4999, 1030, 2), (7001, 1030, 5),
                                      (7001, 1030, 7), (3000, 8200, 5), (6000, 64, 1500), (6000, 64, 1), (1025, 2048, 2), (2049, 40, 2)])
def test_rows_of_the_gate_across_groups_of_tokens(t, h, rows, dtype):
    ins, out = _backward(t, h, dtype, rows, -(-t // rows), seed=1)
    _check(ins, out, rows)

"""Norms that 64 bits hold and 32 do not."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_finite_norm_beyond_fp32_clips_and_does_not_read_as_infinite(dtype):
    """An infinite norm_coef[0] says that an element was not finite and that nothing was clipped: neither holds here."""
    g = torch.full((40, 30), 3e38, dtype=dtype)
    norm = math.sqrt(float((g.double() ** 2).sum()))
    assert norm > torch.finfo(torch.float32).max
    nc = torch.zeros(2, device="cuda")
    t = edgc.Tensor(g.cuda(), torch.full_like(g, 7.0, device="cuda"))
    ctx().grad_sumsq_batch([t])
    ctx().clip_batch([t], 1e30, nc)
    coef = 1e30 / norm
    assert float(nc[0]) == torch.finfo(torch.float32).max
    assert abs(float(nc[1]) - coef) <= 2.0 ** -23 * coef
    want = g.double() * coef
    # the coefficient rounded to fp32, the product to fp32 and to the type
    assert bool(((t.grad_out.cpu().double() - want).abs() <= (2.0 ** -22 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) * want).all())

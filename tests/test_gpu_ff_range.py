"""Kept projections up to the largest numbers of either type: activations and derivatives whose inner powers overflow."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from gpu_util import ctx
from test_gpu_ff import ACTS, _backward_check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ACTS)
def test_projections_up_to_the_largest_numbers(dtype, act):
    """|z| from 1e12 to 3e38: z^2 and z^3 overflow from 1.8e19 and 7e12 on, the activation and its derivative do not.  (The other
    projection is small, so that no output overflows.)"""
    t, h, f = 54, 64, 128
    d = _inputs(t, h, f, dtype, seed=11)
    size = 10.0 ** torch.linspace(12, 38.47, t // 2, dtype=torch.float64)
    sign = torch.tensor([1.0, -1.0], dtype=torch.float64)
    d["gate"] = (size[:, None] * sign).view(t, 1).expand(t, f).to(dtype).contiguous()
    d["up"] = (d["up"].float() * 1e-3).to(dtype)
    v = {k: a.cuda() for k, a in d.items()}
    c = ctx()
    c.reserve_ff(dtype, t, h, f, backward=True)
    out = {"d" + k: torch.full_like(v[k], 7.0) for k in ("x", "w_gate", "w_up", "w_down")}
    c.ff_backward(edgc.FeedForward(v["w_gate"], v["w_up"], v["w_down"], act), v["x"], v["gate"], v["up"], v["dy"], out["dx"],
                  out["dw_gate"], out["dw_up"], out["dw_down"])
    for k, o in out.items():
        assert bool(torch.isfinite(o).all()), k
    _backward_check(d, act, out)

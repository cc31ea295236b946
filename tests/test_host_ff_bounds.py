"""The bounds that the feed-forward block's products are held to on the GPU, on the CPU: they accept outputs that are rounded as the
kernels round them, and none that lacks a share of a sum."""
import pytest
import torch

import test_gpu_ff_products as p


def _outputs(d, act, dtype):
    """The block's outputs in 64 bits but for the roundings: A, dG, dU and every output to the type."""
    q = {k: v.double() for k, v in d.items()}
    r = lambda m: m.to(dtype).double()
    a, da = p._act64(act, q["gate"])
    dA = q["dy"] @ q["w_down"]
    A, dG, dU = r(a * q["up"]), r(dA * q["up"] * da), r(dA * a)
    G, U = q["x"] @ q["w_gate"].t(), q["x"] @ q["w_up"].t()
    Y = r(p._act64(act, G)[0] * U)
    return q, A, dG, dU, G, U, Y


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,h,f", [(700, 1024, 550), (16, 512, 2048), (130, 320, 200), (33, 64, 64), (5, 640, 1536)])
def test_rounded_outputs_pass_and_damaged_ones_do_not(t, h, f, dtype):
    d = p._inputs(t, h, f, dtype, 1, device="cpu")
    act = p.ACTS[(t + h + f) % 3]
    q, A, dG, dU, G, U, Y = _outputs(d, act, dtype)
    good = {"dx": dG @ q["w_gate"] + dU @ q["w_up"], "dw_gate": dG.t() @ q["x"], "dw_up": dU.t() @ q["x"], "dw_down": q["dy"].t() @ A}
    y = Y @ q["w_down"].t()
    p._backward_check(d, act, {k: v.to(dtype) for k, v in good.items()})
    p._forward_check(d, act, y.to(dtype), G.to(dtype), U.to(dtype))
    last_k, last_t = max(0, f - 64), t - max(1, t // 22)
    bad = [("dx", good["dx"] - dU @ q["w_up"]), ("dx", good["dx"] - dG @ q["w_gate"]), ("dw_gate", 0.8 * good["dw_gate"]),
           ("dw_gate", dG[:last_t].t() @ q["x"][:last_t]), ("dw_up", dU[:last_t].t() @ q["x"][:last_t]),
           ("dw_down", q["dy"][:last_t].t() @ A[:last_t]), ("dx", dG[:, :last_k] @ q["w_gate"][:last_k] + dU @ q["w_up"]),
           ("dx", 1.05 * good["dx"]), ("dw_down", good["dw_down"].roll(1, 0))]
    for k, v in bad:
        with pytest.raises(AssertionError):
            p._backward_check(d, act, {n: (v if n == k else g).to(dtype) for n, g in good.items()})
    for v in (Y[:, :last_k] @ q["w_down"][:, :last_k].t(), 0.95 * y, y.roll(1, 1)):
        with pytest.raises(AssertionError):
            p._forward_check(d, act, v.to(dtype))
    with pytest.raises(AssertionError):
        p._forward_check(d, act, y.to(dtype), G.to(dtype), (q["x"][:, 16:] @ q["w_up"][:, 16:].t()).to(dtype))

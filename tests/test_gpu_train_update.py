"""The training example's update of the weights, against the same in 64 bits: clipped gradients, momentum, of the blocks' matrices orthogonalised."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import train_block as tb

pytestmark = pytest.mark.gpu


def newton_schulz(v):
    tall = v.shape[0] > v.shape[1]
    x = v.t() if tall else v
    x = x / (x.norm() + 1e-7)
    for _ in range(5):
        a = x @ x.t()
        x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
    return x.t() if tall else x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("orthogonal", [True, False])
def test_weights_after_two_updates(orthogonal, dtype):
    """Every weight is w - lr v, v = momentum v + the clipped gradient, and of the blocks' matrices the orthogonalised v times sqrt(max(1, rows / columns)).  In the
    type's half steps: the clipped gradient's rounding and two of v, of which directions a third of the mean have three times as much beside them, and lr times
    the update: at most eight of what the weight is moved by; and the weight's own, twice."""
    ctx = edgc.Context(0, max_bins=64, max_rank=max(tb.RANKS), max_rows=64, max_cols=64)
    model = tb.Model(ctx, 2, 64, 96, 100, 50, dtype, seed=3, vocab=40)
    step = tb.Step(model, 0.5, 0.25, 0.9, orthogonal=orthogonal)
    g = torch.Generator().manual_seed(9)
    pairs = model.parameters()
    w, v = [p.double().cpu() for p, _ in pairs], [torch.zeros(p.shape, dtype=torch.float64) for p, _ in pairs]
    before = [x.clone() for x in w]
    matrices = {id(b[k]) for b in model.blocks for k in ("w_gate", "w_up", "w_down")}
    for _ in range(2):
        for _, grad in pairs:
            grad.copy_(torch.randn(grad.shape, generator=g))
        grads = [grad.double().cpu() for _, grad in pairs]
        norm = math.sqrt(sum(float(x.square().sum()) for x in grads))
        step.update(0)
        for i, (p, _) in enumerate(pairs):
            v[i] = 0.9 * v[i] + grads[i] * min(1.0, 0.5 / norm)
            turned = orthogonal and id(p) in matrices
            w[i] -= 0.25 * (math.sqrt(max(1.0, p.shape[0] / p.shape[1])) * newton_schulz(v[i]) if turned else v[i])
    torch.cuda.synchronize()
    half = torch.finfo(dtype).eps / 2
    assert len(matrices) == 6 and len(pairs) > 12
    for (p, _), want, was in zip(pairs, w, before):
        moved = (want - was).norm()
        err = (p.double().cpu() - want).norm()
        assert float(err) <= 8 * max(half, 1e-6) * float(moved) + 2 * half * float(want.norm()), (tuple(p.shape), float(err / moved))
        # and the update is what moves it (as far as roundings to bf16 let a weight of one be moved by less than half their step)
        assert float((p.double().cpu() - was).norm()) >= 0.5 * float(moved) - 2 * half * float(want.norm())
    ctx.close()

"""The stack of blocks with so few tokens that the forward products are those that stream the weights."""
import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import train_block as tb
from test_gpu_train_block import _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,sequence", [(1, 1), (12, 5), (40, 16), (64, 64)])
def test_gradients_through_a_stack_of_blocks(tokens, sequence):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    model = tb.Model(ctx, 3, 96, 160, tokens, sequence, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(tokens, 96, generator=g, device="cuda")
    dn = 1e-2 * torch.randn(tokens, 96, generator=g, device="cuda")
    out = model.forward(x)
    dx = model.backward(dn)
    want, grads, want_dx = _reference(model, x, dn)
    # fp32 through three blocks of two products and two norms each: some hundred units of 2^-23 in the norm
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert rel(out, want) < 300 * 2.0 ** -23 and rel(dx, want_dx) < 300 * 2.0 ** -23
    for (_, got), w in zip(model.parameters(), grads):
        assert rel(got, w) < 300 * 2.0 ** -23
    ctx.close()

"""The norms of queries and keys where there is no head of keys."""
import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [0, 1, 9, 1500])
def test_a_weight_of_no_heads_has_a_gradient_of_zeros(tokens, dtype):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    g = torch.Generator().manual_seed(1)
    randn = lambda *s: torch.randn(s, generator=g).to(dtype).cuda()
    q, dq_out, w_q, w_k, none = randn(tokens, 3, 16), randn(tokens, 3, 16), randn(16), randn(16), torch.empty(tokens, 0, 16, dtype=dtype, device="cuda")
    out = [[torch.full_like(q, 7.0), torch.full_like(w_q, 7.0), torch.full_like(w_k, 7.0)] for _ in range(2)]
    ctx.reserve_qk_norm(max(tokens, 1), 3, 0, 16)
    ctx.qk_norm_forward(q, none, w_q, w_k, None, None, torch.empty_like(q), none)
    ctx.qk_norm_backward(dq_out, none, q, none, w_q, w_k, None, None, out[0][0], none, out[0][1], out[0][2])
    ctx.qk_norm_backward(dq_out, None, q, None, w_q, None, None, None, out[1][0], None, out[1][1], None)
    torch.cuda.synchronize()
    ctx.close()
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    assert bool((out[0][2] == 0).all())

"""The embedding of tokens on both sides of what is written past the caches."""
import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, hidden", [(torch.float32, 2049), (torch.bfloat16, 4097), (torch.bfloat16, 4096)])
@pytest.mark.parametrize("tokens", [16384, 16300, 17000])
def test_rows_of_more_and_less_than_the_caches_are_the_tables(tokens, dtype, hidden):
    """2^27 bytes are 16384 rows of 2048 fp32 or 4096 bf16: one element more, and fewer and more tokens, into rows that are not aligned."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    table = torch.randn(300, hidden, device="cuda", generator=g).to(dtype)
    ids = torch.randint(-2, 302, (tokens,), device="cuda", generator=g)
    wide = torch.full((tokens, hidden + 3), 7.0, dtype=dtype, device="cuda")
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.embed_forward(table, ids, wide[:, 1:1 + hidden])
    torch.cuda.synchronize()
    ctx.close()
    inside = (ids >= 0) & (ids < 300)
    assert torch.equal(wide[:, 1:1 + hidden], table[ids.clamp(0, 299)] * inside[:, None])
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 1 + hidden:] == 7.0).all())

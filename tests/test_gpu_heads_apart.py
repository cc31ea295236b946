"""Heads that are written are refused where they overlap, however far apart their strides would be."""
import pytest

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import binding as b

pytestmark = pytest.mark.gpu


def test_a_span_beyond_64_bits_is_an_overlap():
    """2^31 tokens so far apart that the last one's offset, cut to 64 bits, lies before the next head."""
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    L, tokens, dim = edgc.load_library(), 2 ** 31, 8
    far = 2 ** 40
    refused = 0
    for turn in range(1, 100):
        token = -(-turn * 2 ** 64 // (tokens - 1))
        if ((tokens - 1) * token + dim) % 2 ** 64 > far or token > far:
            continue
        q, out = b._pack_heads(4096, 8, 2 ** 34), b._pack_heads(4096, token, far)
        rc = L.edgc_qk_norm_forward(ctx._h, 0, tokens, 2, 0, dim, q, None, 4096, None, None, 8, None, 0, 0, 1e-6, out, None, None)
        assert rc == b.EINVAL
        refused += 1
    ctx.close()
    assert refused > 10

"""Arguments of the block operators that the binding has to refuse or take before the library sees them (no GPU is needed)."""
import types

import pytest
import torch

import paper_2511_10333_amd as edgc

STREAM = types.SimpleNamespace(cuda_stream=0)


def _no_context():
    """A Context whose library calls all answer EDGC_EINVAL, since it has no handle."""
    c = object.__new__(edgc.Context)
    c._L, c._h = edgc.load_library(), None
    return c


def test_tokens_and_widths_beyond_32_bits_are_refused_not_cut():
    """The library's own limits come after the arguments' 32 bits: 2^32 + 16 tokens are not 16."""
    c, many = _no_context(), 2 ** 32 + 16
    w = edgc.FeedForward(torch.zeros(8, 8), torch.zeros(8, 8), torch.zeros(8, 8))
    m = lambda rows, cols: torch.empty((rows, cols), device="meta")
    x, k = m(many, 8), m(many, 8)
    with pytest.raises(ValueError, match="2\\^32"):
        c.ff_forward(w, x, x, stream=STREAM)
    with pytest.raises(ValueError, match="2\\^32"):
        c.ff_backward(w, x, k, k, x, x, *w.weights, stream=STREAM)
    for reserve in ((many, 8, 8), (8, many, 8), (8, 8, many), (-1, 8, 8)):
        with pytest.raises(ValueError, match="2\\^32"):
            c.reserve_ff(torch.float32, *reserve)
    for reserve in ((many, 8), (8, many), (-1, 8)):
        with pytest.raises(ValueError, match="2\\^32"):
            c.reserve_block_norm(*reserve)
    with pytest.raises(ValueError, match="2\\^32"):
        edgc.FeedForward(m(many, 8), m(many, 8), m(8, many))
    with pytest.raises(ValueError, match="2\\^32"):
        edgc.FeedForward(m(8, many), m(8, many), m(many, 8))
    with pytest.raises(edgc.EdgcError):                     # what fits is handed on
        c.ff_forward(w, torch.zeros(4, 8), torch.zeros(4, 8), stream=STREAM)


def test_rows_per_gate_beyond_64_bits_is_refused_not_cut():
    """2^64 + 3 tokens per row of the gate are one row for all of them, and not one for every three."""
    c = _no_context()
    x, v, g = torch.zeros(9, 8), torch.zeros(8), torch.zeros(1, 8)
    r = torch.zeros(9)
    with pytest.raises(ValueError, match="rows_per_gate"):
        c.block_norm_forward(x, x, v, g, v, x, x, rows_per_gate=2 ** 64 + 3, stream=STREAM)
    with pytest.raises(ValueError, match="rows_per_gate"):
        c.block_norm_backward(x, x, x, x, v, g, v, r, r, x, x, v, g, v, rows_per_gate=2 ** 64 + 3, stream=STREAM)
    with pytest.raises(edgc.EdgcError):                     # what fits is handed on
        c.block_norm_forward(x, x, v, g, v, x, x, rows_per_gate=2 ** 64 - 1, stream=STREAM)


def test_the_row_stride_of_a_single_row_does_not_count():
    """One token's projections may lie in buffers of different widths, and a single row may have any stride."""
    c = _no_context()
    w = edgc.FeedForward(torch.zeros(12, 8), torch.zeros(12, 8), torch.zeros(8, 12))
    x, gate, up = torch.zeros(1, 8), torch.zeros(1, 12), torch.zeros(1, 20)[:, :12]
    up = up.as_strided((1, 12), (20, 1))
    with pytest.raises(edgc.EdgcError):                     # handed on, and refused for want of a context alone
        c.ff_forward(w, x, x.clone(), gate, up, stream=STREAM)
    with pytest.raises(edgc.EdgcError):
        c.ff_backward(w, x, gate, up, x, x.clone(), *w.weights, stream=STREAM)
    far = torch.zeros(12, dtype=torch.bfloat16).as_strided((1, 12), (2 ** 41, 1))
    one = edgc.FeedForward(far, far, torch.zeros(12, 1, dtype=torch.bfloat16))
    assert (one.c.ld_gate, one.c.ld_up, one.c.ld_down) == (12, 12, 1)
    with pytest.raises(ValueError):                         # of two rows it does
        c.ff_forward(w, torch.zeros(2, 8), torch.zeros(2, 8), torch.zeros(2, 12), torch.zeros(2, 20)[:, :12], stream=STREAM)

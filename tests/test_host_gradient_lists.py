"""What a list of gradients has to be before its descriptors reach the library (descriptors are built without a GPU)."""
import pytest
import torch

import paper_2511_10333_amd as edgc


def _one(grad, grad_out=None):
    return edgc.PreparedBatch([edgc.Tensor(grad, grad if grad_out is None else grad_out)]).arr[0]


def test_sizes_beyond_the_descriptors_fields_are_refused_not_cut():
    """m and n are 32 bits wide: a flat gradient of 2^32 + 5 elements is not one of five."""
    with pytest.raises(ValueError, match="2\\^32"):
        _one(torch.empty(2 ** 32 + 5, dtype=torch.bfloat16, device="meta"))
    with pytest.raises(ValueError, match="2\\^32"):
        _one(torch.empty((2 ** 32, 2), dtype=torch.bfloat16, device="meta"))
    with pytest.raises(ValueError, match="2\\^32"):
        _one(torch.empty((2, 2 ** 32 + 1), device="meta"))
    d = _one(torch.empty(2 ** 32 - 1, dtype=torch.bfloat16, device="meta"))
    assert (d.m, d.n) == (1, 2 ** 32 - 1)
    d = _one(torch.empty((2 ** 20, 2 ** 13), device="meta"))
    assert (d.m, d.n, d.ld) == (2 ** 20, 2 ** 13, 2 ** 13)

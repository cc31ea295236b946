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


def test_views_whose_neighbours_are_not_neighbours_in_memory_are_refused():
    """The library reads rows of adjacent elements: a column of a matrix, or a transposed one, is not that."""
    g = torch.zeros(10, 4)
    for bad in (g[:, 0], g.t(), g[:, ::2], g.view(-1)[::2], torch.zeros(1).expand(10), g.t()[:1]):
        with pytest.raises(ValueError, match="contiguous rows"):
            _one(bad)
        with pytest.raises(ValueError, match="contiguous rows"):
            _one(torch.zeros(bad.shape), bad)
    for bad in (g.view(2, 5, 4), torch.zeros(())):
        with pytest.raises(ValueError):
            _one(bad)
    d = _one(g[:, 1:3])                                     # columns of a wider buffer
    assert (d.m, d.n, d.ld, d.ld_out) == (10, 2, 4, 4)
    d = _one(g[:, :1], g[:, 1:2])
    assert (d.m, d.n, d.ld) == (10, 1, 4)
    d = _one(g.t()[:, :1])                                  # a column as a matrix: nothing lies beside its elements' rows
    assert (d.m, d.n, d.ld) == (4, 1, 1)
    d = _one(g[3], g[4])
    assert (d.m, d.n) == (1, 4)
    d = _one(g.view(-1)[5:6:3])                             # one element
    assert (d.m, d.n) == (1, 1)


def test_an_output_of_another_type_or_size_is_refused():
    """grad_out is written as a matrix of the gradient's type and shape: anything narrower or shorter would be written past its end."""
    g = torch.zeros(6, 8)
    for bad in (torch.zeros(6, 8).bfloat16(), torch.zeros(6, 8).double()):
        with pytest.raises(TypeError, match="grad_out"):
            _one(g, bad)
    with pytest.raises(TypeError, match="grad_out"):
        _one(g.bfloat16(), g)
    for bad in (torch.zeros(5, 8), torch.zeros(6, 7), torch.zeros(8, 6), torch.zeros(48), torch.zeros(6), torch.zeros(0)):
        with pytest.raises(ValueError, match="grad_out"):
            _one(g, bad)
    with pytest.raises(ValueError, match="grad_out"):
        _one(torch.zeros(9), torch.zeros(8))
    with pytest.raises(ValueError, match="grad_out"):
        _one(torch.zeros(9), torch.zeros(9, 1))
    assert _one(torch.zeros(9), torch.zeros(1, 9)).n == 9           # one row either way
    assert edgc.PreparedBatch([edgc.Tensor(None, g)]).arr[0].m == 6
    assert edgc.PreparedBatch([edgc.Tensor(g, None)]).arr[0].grad_out is None

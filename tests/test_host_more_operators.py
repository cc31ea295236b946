"""Arguments of the operators before and after the stack of blocks that are refused before anything could run (no GPU is needed)."""
import types

import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import binding as b

STREAM = types.SimpleNamespace(cuda_stream=0)


def _no_context():
    """A Context whose library calls all answer EDGC_EINVAL, since it has no handle."""
    c = object.__new__(edgc.Context)
    c._L, c._h, c.device = edgc.load_library(), None, 0
    return c


def test_orthogonalize_without_a_context_or_with_sizes_beyond_its_fields():
    L = edgc.load_library()
    assert L.edgc_reserve_orthogonalize(None, 0, None, None, 0, 5) == b.EINVAL
    assert L.edgc_orthogonalize_batch(None, None, 0, 0, 5, 1.0, 0.0, 0.0, 0.0, None, None) == b.EINVAL
    c = _no_context()
    t = [edgc.Tensor(torch.zeros(4, 4), torch.zeros(4, 4))]
    with pytest.raises(edgc.EdgcError):                     # what fits is handed on
        c.orthogonalize_batch(t, stream=STREAM)
    for steps in (-1, 2 ** 32 + 5):
        with pytest.raises(ValueError, match="2\\^32"):
            c.orthogonalize_batch(t, steps=steps, stream=STREAM)
        with pytest.raises(ValueError, match="2\\^32"):
            c.reserve_orthogonalize(torch.float32, [(4, 4)], steps)
    with pytest.raises(ValueError, match="2\\^32"):
        c.reserve_orthogonalize(torch.float32, [(4, 2 ** 32 + 4)])
    with pytest.raises(TypeError):
        c.reserve_orthogonalize(torch.float16, [(4, 4)])
    with pytest.raises(ValueError, match="scales"):
        c.orthogonalize_batch(t, scales=[1.0, 2.0], stream=STREAM)

"""Arguments of the operators before and after the stack of blocks that are refused before anything could run (no GPU is needed)."""
import os
import subprocess
import types

import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


def test_tiles_of_a_symmetric_output_begin_inside_it_and_cover_its_lower_half_once(tmp_path):
    """Tiles twice as high as wide: of the last row of tiles the last one can begin beyond the matrix, and is not to be made."""
    src = tmp_path / "tiles.cpp"
    src.write_text('#include <cstdio>\n#include "ortho_tiles.h"\n'
                   'using namespace edgc;\n'
                   'template <unsigned R> void go(unsigned n, unsigned bm) { unsigned bn = bm / R, m = (n + bm - 1) / bm, k = (n + bn - 1) / bn;\n'
                   '  for (unsigned id = 0; id < ortho_tiles<R>(m, k); ++id) { unsigned tm, tn; ortho_tile_of<R>(id, m, k, tm, tn);\n'
                   '    std::printf("%u %u %u %u %u\\n", n, bm, bn, tm * bm, tn * bn); } }\n'
                   'int main() { for (unsigned n = 32; n <= 7200; n = n < 1200 ? n + 32 : n + 480) { go<2>(n, 256); go<1>(n, 256); go<1>(n, 128); } }\n')
    exe = tmp_path / "tiles"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2511_10333_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    seen = {}
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        n, bm, bn, m0, n0 = map(int, line.split())
        assert m0 < n and n0 < n, line
        at = seen.setdefault((n, bm, bn), set())
        assert (m0, n0) not in at, line
        at.add((m0, n0))
    for (n, bm, bn), at in seen.items():
        # every tile that has a square of 32 on or below the diagonal, and no other
        assert at == {(m, c) for m in range(0, n, bm) for c in range(0, n, bn) if c < m + bm}, (n, bm, bn)

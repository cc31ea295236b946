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
    for batch in (t, edgc.PreparedBatch(t)):                # host memory is not handed to a kernel
        with pytest.raises(ValueError, match="device"):
            c.orthogonalize_batch(batch, stream=STREAM)
    c.device = -1                                           # (host tensors count as the context's)
    for batch in (t, edgc.PreparedBatch(t)):
        with pytest.raises(edgc.EdgcError):                 # what fits is handed on
            c.orthogonalize_batch(batch, stream=STREAM)
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
    src = tmp_path / "tiles.cpp"
    src.write_text('#include <cstdio>\n#include "ortho_tiles.h"\n'
                   'using namespace edgc;\n'
                   'void go(unsigned n, unsigned bm) { const unsigned m = (n + bm - 1) / bm;\n'
                   '  for (unsigned id = 0; id < ortho_tiles(m); ++id) { unsigned tm, tn; ortho_tile_of(id, m, tm, tn);\n'
                   '    std::printf("%u %u %u %u\\n", n, bm, tm * bm, tn * bm); } }\n'
                   'int main() { for (unsigned n = 32; n <= 7200; n = n < 1200 ? n + 32 : n + 480) { go(n, 256); go(n, 128); go(n, 64); } }\n')
    exe = tmp_path / "tiles"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2511_10333_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    seen = {}
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        n, bm, m0, n0 = map(int, line.split())
        assert m0 < n and n0 < n, line
        at = seen.setdefault((n, bm), set())
        assert (m0, n0) not in at, line
        at.add((m0, n0))
    for (n, bm), at in seen.items():
        # every tile that has a square of 32 on or below the diagonal, and no other
        assert at == {(m, c) for m in range(0, n, bm) for c in range(0, m + 1, bm)}, (n, bm)


def _meta(*shape, dtype=torch.float32):
    return torch.empty(shape, device="meta", dtype=dtype)


def test_tensors_that_the_gpu_cannot_read_are_refused():
    """Host memory, or another GPU's, is not handed to a kernel."""
    c = _no_context()
    table, ids, out = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8)
    with pytest.raises(ValueError, match="device"):
        c.embed_forward(table, ids, out, stream=STREAM)
    with pytest.raises(ValueError, match="device"):
        c.embed_backward(ids, out, table, stream=STREAM)
    q, w = torch.zeros(3, 2, 8), torch.ones(8)
    with pytest.raises(ValueError, match="device"):
        c.qk_norm_forward(q, None, w, None, None, None, q, None, stream=STREAM)
    with pytest.raises(ValueError, match="device"):
        c.qk_norm_backward(q, None, q, None, w, None, None, None, q, None, w, None, stream=STREAM)


def test_embed_without_a_context_and_with_what_it_does_not_take():
    L = edgc.load_library()
    assert L.edgc_embed_forward(None, 0, None, 0, 1, 1, None, 8, 0, 0, 1.0, None, 0, None) == b.EINVAL
    assert L.edgc_reserve_embed(None, 1, 1, 1) == b.EINVAL
    assert L.edgc_embed_backward(None, 0, None, 8, 0, 0, None, 0, 1, 1, 1.0, None, 0, 0, None) == b.EINVAL
    c = _no_context()
    c.device = -1
    table, ids, out = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8)
    with pytest.raises(edgc.EdgcError):                     # what fits is handed on
        c.embed_forward(table, ids, out, stream=STREAM)
    with pytest.raises(edgc.EdgcError):
        c.embed_backward(ids.int(), out, table, stream=STREAM)
    for bad in (ids.double(), ids.short(), ids.bool()):
        with pytest.raises(TypeError, match="ids"):
            c.embed_forward(table, bad, out, stream=STREAM)
    with pytest.raises(ValueError, match="ids"):
        c.embed_forward(table, torch.zeros(3, 2, dtype=torch.int64)[:, 0], out, stream=STREAM)
    with pytest.raises(ValueError, match="ids"):
        c.embed_forward(table, ids.view(3, 1), out, stream=STREAM)
    with pytest.raises(ValueError, match="out"):
        c.embed_forward(table, ids, torch.zeros(4, 8), stream=STREAM)
    with pytest.raises(TypeError, match="out"):
        c.embed_forward(table, ids, out.bfloat16(), stream=STREAM)
    with pytest.raises(ValueError, match="dy"):
        c.embed_backward(ids, torch.zeros(8, 3).t(), table, stream=STREAM)
    with pytest.raises(ValueError, match="first_id"):
        c.embed_forward(table, ids, out, first_id=2 ** 63, stream=STREAM)
    with pytest.raises(TypeError):
        c.embed_forward(table.double(), ids, out.double(), stream=STREAM)
    for sizes in ((2 ** 32 + 1, 4, 4), (4, 2 ** 32 + 1, 4), (4, 4, 2 ** 32 + 1), (-1, 4, 4)):
        with pytest.raises(ValueError, match="2\\^32"):
            c.reserve_embed(*sizes)
    with pytest.raises(ValueError, match="2\\^32"):
        c.embed_forward(_meta(2 ** 32 + 1, 8), ids, out, stream=STREAM)


def test_qk_norm_without_a_context_and_with_what_it_does_not_take():
    L = edgc.load_library()
    assert L.edgc_reserve_qk_norm(None, 1, 1, 1, 1) == b.EINVAL
    assert L.edgc_qk_norm_forward(None, 0, 0, 1, 0, 1, *[None] * 5, 8, None, 0, 0, 0.0, None, None, None) == b.EINVAL
    assert L.edgc_qk_norm_backward(None, 0, 0, 1, 0, 1, *[None] * 7, 8, None, 0, 0, 0.0, *[None] * 5) == b.EINVAL
    c = _no_context()
    c.device = -1
    q, k, w, pos, f = torch.zeros(3, 4, 8), torch.zeros(3, 2, 8), torch.ones(8), torch.arange(3), torch.ones(4, dtype=torch.float64)
    with pytest.raises(edgc.EdgcError):                     # what fits is handed on
        c.qk_norm_forward(q, k, w, w, pos, f, q, k, stream=STREAM)
    with pytest.raises(edgc.EdgcError):
        c.qk_norm_forward(q, None, w, None, None, None, q, None, stream=STREAM)
    fwd = lambda *a: c.qk_norm_forward(*a, stream=STREAM)
    for bad, kind in (((q, k, w, w, pos, f.float(), q, k), TypeError), ((q, k, w, w, pos.double(), f, q, k), TypeError), ((q, k, w, w, pos[:2], f, q, k), ValueError),
                      ((q, k, w, w, None, f, q, k), ValueError), ((q, k, w, None, pos, f, q, k), ValueError), ((q, k, w, w, pos, f, q, None), ValueError),
                      ((q, None, w, None, pos, f, q, k), ValueError), ((q, k, w[:7], w, pos, f, q, k), ValueError), ((q, k, w, w.bfloat16(), pos, f, q, k), TypeError),
                      ((q, k.bfloat16(), w, w, pos, f, q, k), TypeError), ((q, torch.zeros(2, 2, 8), w, w, pos, f, q, k), ValueError),
                      ((q, k, w, w, pos, f, torch.zeros(3, 8, 4).transpose(1, 2), k), ValueError), ((q[0], k, w, w, pos, f, q, k), ValueError)):
        with pytest.raises(kind):
            fwd(*bad)
    with pytest.raises(ValueError):
        c.qk_norm_backward(q, k, q, k, w, w, pos, f, q, k, w, torch.ones(16)[::2], stream=STREAM)
    for sizes in ((2 ** 32 + 1, 4, 4, 4), (4, 2 ** 32 + 1, 4, 4), (4, 4, -1, 4), (4, 4, 4, 2 ** 32 + 1)):
        with pytest.raises(ValueError, match="2\\^32"):
            c.reserve_qk_norm(*sizes)


def test_the_heads_descriptor_agrees_with_the_header(tmp_path):
    src = tmp_path / "heads.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "edgc.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu\\n", sizeof(edgc_heads), offsetof(edgc_heads, p), offsetof(edgc_heads, token), offsetof(edgc_heads, head));'
                   ' return 0; }\n')
    exe = tmp_path / "heads"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    sizes = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    packed = b._pack_heads(0x1122334455667788, 3, 5)
    assert sizes == [len(packed), 0, 8, 16]
    assert [int.from_bytes(packed[at:at + 8], "little") for at in sizes[1:]] == [0x1122334455667788, 3, 5]

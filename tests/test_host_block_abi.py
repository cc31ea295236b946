"""CPU-side checks of the block operators' entry points: what the header declares, and what a call without a context returns."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2511_10333_amd as edgc
from paper_2511_10333_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_and_enum_agree_with_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "edgc.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(edgc_ff), offsetof(edgc_ff, ld_gate), offsetof(edgc_ff, hidden),'
                   ' offsetof(edgc_ff, dtype), offsetof(edgc_ff, act)); printf("%d %d %d\\n", EDGC_SILU, EDGC_GELU, EDGC_GELU_TANH); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    first, second = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    f = b._FF
    assert [int(x) for x in first.split()] == [ctypes.sizeof(f), f.ld_gate.offset, f.hidden.offset, f.dtype.offset, f.act.offset]
    assert [int(x) for x in second.split()] == [b.ACTIVATIONS[k] for k in ("silu", "gelu", "gelu_tanh")]


def test_calls_without_a_context_are_refused():
    L = edgc.load_library()
    assert L.edgc_grad_sumsq_batch(None, None, 0, 0, 0, None, None) == b.EINVAL
    assert L.edgc_clip_batch(None, None, 0, 0, 1.0, None, None, None) == b.EINVAL
    assert L.edgc_reserve_block_norm(None, 1, 1) == b.EINVAL
    assert L.edgc_reserve_ff(None, 0, 1, 1, 1, 0) == b.EINVAL
    assert L.edgc_ff_forward(None, None, None, 0, 1, None, 0, None, None, 0, None) == b.EINVAL
    assert L.edgc_block_norm_forward(None, 0, 1, 1, *[None] * 4, 0, None, 1.0, 0.0, *[None] * 5) == b.EINVAL


def test_descriptor_of_a_feed_forward_block():
    wide = torch.zeros(12, 20)
    w = edgc.FeedForward(wide[:, :8], torch.zeros(12, 8), torch.zeros(8, 12), "gelu")
    assert (w.hidden, w.ff, w.c.ld_gate, w.c.ld_up, w.c.ld_down, w.c.act, w.c.dtype) == (8, 12, 20, 8, 12, 1, b.F32)
    one = edgc.FeedForward(torch.zeros(1, 8, dtype=torch.bfloat16), torch.zeros(1, 8, dtype=torch.bfloat16), torch.zeros(8, 1, dtype=torch.bfloat16))
    assert (one.c.ld_gate, one.c.ld_down, one.c.dtype) == (8, 1, b.BF16)
    with pytest.raises(ValueError):
        edgc.FeedForward(torch.zeros(12, 8), torch.zeros(12, 8), torch.zeros(12, 8))
    with pytest.raises(ValueError):
        edgc.FeedForward(torch.zeros(1, 8).expand(12, 8), torch.zeros(12, 8), torch.zeros(8, 12))      # rows that overlap
    with pytest.raises(TypeError):
        edgc.FeedForward(torch.zeros(12, 8).double(), torch.zeros(12, 8).double(), torch.zeros(8, 12).double())

"""Reservations of the block operators: what a later one replaces, and what it leaves in place."""
import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu


def _block(ctx, t, h, f, dtype, seed):
    """Forward and backward of one block; what it computes, and a call that computes it again."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0: (std * torch.randn(*s, generator=g, device="cuda")).to(dtype)
    wg, wu, wd, w = r(f, h, std=h ** -0.5), r(f, h, std=h ** -0.5), r(h, f, std=f ** -0.5), r(h)
    ff = edgc.FeedForward(wg, wu, wd)
    x, dn, e = r(t, h), r(t, h, std=1e-2), lambda *s: torch.empty(*s, device="cuda", dtype=dtype)
    y, gate, up, n, xo = e(t, h), e(t, f), e(t, f), e(t, h), e(t, h)
    r1, r2 = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    dx, dy, dwp, dwn, dxi, dw = e(t, h), e(t, h), e(h), e(h), e(t, h), [e(f, h), e(f, h), e(h, f)]

    def go():
        ctx.ff_forward(ff, x, y, gate, up)
        ctx.block_norm_forward(x, y, w, None, w, xo, n, r1, r2)
        ctx.block_norm_backward(dn, dn, xo, y, w, None, w, r1, r2, dx, dy, dwp, None, dwn)
        ctx.ff_backward(ff, x, gate, up, dy, dxi, *dw)
    return go, [y, n, dx, dy, dwp, dwn, dxi] + dw


def _reserve(ctx, t, h, f, dtype):
    ctx.reserve_ff(dtype, t, h, f, backward=True)
    ctx.reserve_block_norm(t, h)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_smaller_reservation_leaves_a_captured_graph_its_memory(dtype):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    big, small = (300, 192, 520), (40, 64, 100)
    _reserve(ctx, *big, dtype)
    go, out = _block(ctx, *big, dtype, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for sizes in (small, big, (300, 192, 64)):
        _reserve(ctx, *sizes, dtype)
        other, got = _block(ctx, *sizes, dtype, 2)
        other()
        junk = [torch.full((1 << 22,), float("nan"), device="cuda") for _ in range(8)]     # would land in memory that was freed
        for o in out:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        del junk
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_limits_are_those_of_the_last_reservation(dtype):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    sizes = [(40, 64, 100), (300, 192, 520), (40, 64, 100), (200, 320, 64)]
    for s in sizes:
        _reserve(ctx, *s, dtype)
        for q in sizes:
            go, out = _block(ctx, *q, dtype, 3)
            if all(a <= b for a, b in zip(q, s)):
                go()
                torch.cuda.synchronize()
                assert all(bool(torch.isfinite(o).all()) for o in out)
        go, _ = _block(ctx, 400, 400, 600, dtype, 3)
        with pytest.raises(edgc.EdgcError):
            go()
        with pytest.raises(edgc.EdgcError):
            t = torch.zeros(s[0] + 1, s[1], device="cuda", dtype=dtype)
            v, r = torch.ones(s[1], device="cuda", dtype=dtype), torch.ones(s[0] + 1, device="cuda")
            ctx.block_norm_backward(t, t, t, None, None, None, v, None, r, t, None, None, None, v.clone())
    ctx.reserve_ff(dtype, 0, 64, 100)
    ctx.reserve_block_norm(0, 64)
    go, _ = _block(ctx, 40, 64, 100, dtype, 3)
    with pytest.raises(edgc.EdgcError):
        go()
    ctx.close()

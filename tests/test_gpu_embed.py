"""The embedding of tokens and its gradient against 64-bit arithmetic on the host."""
import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    yield c
    c.close()


def randn(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def strided(t, pad, value):
    """The matrix as columns of a wider buffer, on the GPU: (buffer, view)."""
    wide = torch.full((t.shape[0], t.shape[1] + pad + 1), value, dtype=t.dtype, device="cuda")
    view = wide[:, 1:1 + t.shape[1]]
    view.copy_(t)
    return wide, view


def make_ids(kind, tokens, vocab, first, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "same":
        rows = torch.full((tokens,), min(vocab - 1, 3))
    elif kind == "skewed":
        rows = torch.clamp(torch.exp(torch.rand(tokens, generator=g) * torch.log(torch.tensor(vocab + 1.0))).long() - 1, 0, vocab - 1)
    else:
        rows = torch.randint(0, vocab, (tokens,), generator=g)
    ids = rows + first
    if kind == "outside" and tokens:
        away = torch.rand(tokens, generator=g) < 0.4
        ids = torch.where(away, torch.where(torch.rand(tokens, generator=g) < 0.5, first - 1 - rows, first + vocab + rows), ids)
    return ids


def want_backward(ids, dy, vocab, first, scale):
    """Sums in 64 bits, and of the absolute values, with the number of terms."""
    row = ids.long() - first
    inside = (row >= 0) & (row < vocab)
    d = dy.double()[inside]
    sums = torch.zeros(vocab, dy.shape[1], dtype=torch.float64).index_add_(0, row[inside], d) * scale
    sizes = torch.zeros(vocab, dy.shape[1], dtype=torch.float64).index_add_(0, row[inside], d.abs()) * abs(scale)
    return sums, sizes, torch.bincount(row[inside], minlength=vocab).double()


def check_sums(got, sums, sizes, count, dtype, before=None):
    """n fp32 sums are off by less than n 2^-24 of the terms' sizes, the product with the scale (and what is added to) by a rounding, the output by half a step."""
    want = sums if before is None else sums + before.double()
    size = sizes + (0 if before is None else before.double().abs())
    bound = size * (count[:, None] + 3) * 2.0 ** -24 + want.abs() * torch.finfo(dtype).eps / 2 + 1e-40
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("id_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("tokens,vocab,hidden", [(1, 1, 1), (1, 300, 4096), (3, 7, 5), (65, 1000, 513), (130, 40, 2049), (1000, 17, 64)])
def test_forward(ctx, tokens, vocab, hidden, id_type, dtype):
    table, ids = randn((vocab, hidden), 1, dtype), make_ids("outside", tokens, vocab, 50, 2).to(id_type)
    _, t = strided(table, 4, 9.0)
    wide, out = strided(torch.zeros(tokens, hidden, dtype=dtype), 2, 7.0)
    ctx.embed_forward(t, ids.cuda(), out, scale=0.3, first_id=50)
    row = ids.long() - 50
    inside = (row >= 0) & (row < vocab)
    want = torch.where(inside[:, None], table[row.clamp(0, vocab - 1)].double() * torch.tensor(0.3).double(), 0.0)
    err = (out.double().cpu() - want).abs()
    assert bool((err <= want.abs() * (2.0 ** -24 + torch.finfo(dtype).eps / 2)).all())
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 1 + hidden:] == 7.0).all())


BACKWARD = [("uniform", 1, 1, 1), ("uniform", 1, 300, 4096), ("uniform", 3, 7, 5), ("uniform", 2, 1, 9), ("outside", 65, 1000, 513), ("skewed", 130, 40, 2049),
            ("skewed", 5000, 300, 70), ("same", 1000, 17, 64), ("same", 1025, 9, 257), ("outside", 4097, 70000, 8), ("skewed", 3000, 513, 520), ("uniform", 31, 2, 3),
            ("uniform", 2048, 2050, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,tokens,vocab,hidden", BACKWARD)
def test_backward(ctx, kind, tokens, vocab, hidden, accumulate, dtype):
    first = -5 if kind == "outside" else 0
    ids = make_ids(kind, tokens, vocab, first, 3).to(torch.int32 if tokens % 2 else torch.int64)
    dy, before = randn((tokens, hidden), 4, dtype), randn((vocab, hidden), 5, dtype)
    _, d = strided(dy, 3, float("nan"))
    wide, dtable = strided(before, 5, 7.0)
    ctx.reserve_embed(tokens, vocab, hidden)
    ctx.embed_backward(ids.cuda(), d, dtable, scale=0.5, first_id=first, accumulate=accumulate)
    sums, sizes, count = want_backward(ids, dy, vocab, first, 0.5)
    check_sums(dtable, sums, sizes, count, dtype, before if accumulate else None)
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, 1 + hidden:] == 7.0).all())
    if accumulate:
        empty = count == 0
        assert torch.equal(dtable.cpu()[empty], before[empty])


def test_a_large_table_and_many_tokens(ctx):
    """The largest number of rows that a block of the sort takes, and more tokens than one look at them."""
    tokens, vocab, hidden = 70001, 600000, 8
    ids = make_ids("skewed", tokens, vocab, 0, 6)
    ids[::3] = torch.randint(0, vocab, (len(ids[::3]),), generator=torch.Generator().manual_seed(7))
    dy = randn((tokens, hidden), 8, F32)
    dtable = torch.full((vocab, hidden), 3.0, device="cuda")
    ctx.reserve_embed(tokens, vocab, hidden)
    ctx.embed_backward(ids.cuda(), dy.cuda(), dtable)
    check_sums(dtable, *want_backward(ids, dy, vocab, 0, 1.0), F32)


def test_no_tokens(ctx):
    none, d = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, 33, device="cuda")
    table = torch.full((70, 33), 4.0, device="cuda")
    ctx.reserve_embed(0, 70, 33)
    ctx.embed_forward(table, none, d)
    ctx.embed_backward(none, d, table, accumulate=True)
    assert bool((table == 4.0).all())
    ctx.embed_backward(none, d, table)
    assert bool((table == 0.0).all())


def test_rows_beyond_32_bit_offsets(ctx):
    """A table whose last rows begin behind 2^32 elements."""
    vocab, hidden, ld = 4200, 16, 1 << 20
    wide = torch.zeros((vocab, ld), dtype=BF16, device="cuda")
    table = wide[:, :hidden]
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], device="cuda")
    table[-2:] = randn((2, hidden), 9, BF16).cuda()
    out = torch.empty(4, hidden, dtype=BF16, device="cuda")
    ctx.embed_forward(table, ids, out)
    assert torch.equal(out, table[ids])
    dy = randn((4, hidden), 10, BF16)
    ctx.reserve_embed(4, vocab, hidden)
    ctx.embed_backward(ids, dy.cuda(), table)
    check_sums(table, *want_backward(ids.cpu(), dy, vocab, 0, 1.0), BF16)
    assert bool((wide[-1, hidden:] == 0).all())


def test_what_is_not_finite_stays_in_its_row(ctx):
    ids = torch.tensor([2, 1, 2, 3])
    dy = randn((4, 20), 11, F32)
    dy[0, 3], dy[3, 5] = float("nan"), float("inf")
    dtable = torch.empty(6, 20, device="cuda")
    ctx.reserve_embed(4, 6, 20)
    ctx.embed_backward(ids.cuda(), dy.cuda(), dtable)
    bad = ~torch.isfinite(dtable.cpu())
    assert bad.nonzero().tolist() == [[2, 3], [3, 5]]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_same_tokens_give_the_same_bits_also_from_a_graph(ctx, dtype):
    tokens, vocab, hidden = 3000, 500, 200
    ids, dy = torch.zeros(tokens, dtype=torch.int64, device="cuda"), torch.zeros(tokens, hidden, dtype=dtype, device="cuda")
    dtable = torch.empty(vocab, hidden, dtype=dtype, device="cuda")
    ctx.reserve_embed(tokens, vocab, hidden)
    fill = lambda s: (ids.copy_(make_ids("skewed", tokens, vocab, 0, s)), dy.copy_(randn((tokens, hidden), s + 50, dtype)))
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.embed_backward(ids, dy, dtable)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.embed_backward(ids, dy, dtable)
    for s in (1, 2, 3, 1):
        fill(s)
        graph.replay()
        torch.cuda.synchronize()
        replayed = dtable.clone()
        ctx.embed_backward(ids, dy, dtable)
        torch.cuda.synchronize()
        assert torch.equal(replayed, dtable)
        check_sums(dtable, *want_backward(ids.cpu(), dy.cpu(), vocab, 0, 1.0), dtype)


def test_refusals(ctx):
    ids, dy, dt = torch.zeros(10, dtype=torch.int64, device="cuda"), torch.zeros(10, 8, device="cuda"), torch.zeros(20, 8, device="cuda")

    def refused(match, f, *a, **kw):
        with pytest.raises(edgc.EdgcError, match=match) as e:
            f(*a, **kw)
        assert e.value.code == -1
    ctx.reserve_embed(0, 1, 1)
    refused("reserve_embed", ctx.embed_backward, ids, dy, dt)
    ctx.reserve_embed(10, 20, 8)
    ctx.embed_backward(ids, dy, dt)
    refused("reserve_embed", ctx.embed_backward, torch.zeros(1000, dtype=torch.int64, device="cuda"), torch.zeros(1000, 8, device="cuda"), dt)
    for scale in (float("nan"), float("inf")):
        refused("scale", ctx.embed_backward, ids, dy, dt, scale=scale)
        refused("scale", ctx.embed_forward, dt, ids, dy, scale=scale)
    refused("first_id", ctx.embed_forward, dt, ids, dy, first_id=2 ** 62 + 1)
    refused("vocab", ctx.reserve_embed, 1, 2 ** 20 + 1, 8)
    refused("vocab", ctx.reserve_embed, 1, 8, 0)
    refused("tokens", ctx.reserve_embed, 2 ** 26 + 1, 8, 8)
    refused("vocab", ctx.embed_forward, torch.zeros(0, 8, device="cuda"), ids, dy)

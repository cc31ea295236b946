"""The orthogonalised update against the same steps in 64 bits."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

COEFS = (3.4445, -4.7750, 2.0315)
F32, BF16 = torch.float32, torch.bfloat16
SEGMENT = {F32: 3, BF16: 5}         # steps on A between two A = X X^T


def want(g, steps, scale=1.0, eps=1e-7, coefs=COEFS, device="cpu"):
    a, b, c = coefs
    x = g.double().to(device)
    x = x.view(1, -1) if x.dim() == 1 else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        gram = x @ x.t() if x.shape[0] <= x.shape[1] else None
        x = a * x + (b * gram + c * gram @ gram) @ x if gram is not None else a * x + x @ (b * x.t() @ x + c * (x.t() @ x) @ (x.t() @ x))
    return (scale * x).view(g.shape)


def tolerance(shape, steps, dtype):
    """In the norm.  An error d of A_0 relative to its largest value enters W by |b| / a = 1.4 of it, and the next A by a^2 = 12, relative to what
    comes of the smallest singular values: 1.4 (1 + 12 + 144 + ..) d over a segment, as a matrix of such errors (2 / sqrt s of it in the norm, at most
    1).  d is the planes' 2^-22, half of it for the two operands' roundings of either sign, 2^-23.  fp32 sums of l products wander by sqrt(3 l) 2^-25 in
    each of the products of X, some ten of them.  The output is rounded once."""
    s, l = (1, shape[0]) if len(shape) == 1 else (min(shape), max(shape))
    n, segments = min(steps, SEGMENT[dtype]), -(-steps // SEGMENT[dtype])
    carried = 1.4 * sum(12.0 ** k for k in range(n)) * min(1.0, 2 / math.sqrt(s)) * 2.0 ** -23
    return segments * carried + 10 * math.sqrt(3 * l) * 2.0 ** -25 + torch.finfo(dtype).eps / 2


def of_the_input(g, steps):
    """What fp32 gradients' two planes lose, for gradients with singular values far below the largest.  Of 24 significant bits they hold 22 and the
    residual's sign: a last bit that is set is lost where the bit before the residual's is too, a quarter of all, an error of 2^-23 of the element's
    leading bit, 2^-24 in the mean of the squares.  As a matrix of errors of size t = 2^-24 |X| / sqrt(s l) each it changes a direction of singular value
    z by t (sqrt s + sqrt l) / z of itself, and the update, whose singular values are p(z), by that of p(z).  A second X, after two steps of 3.44, has a
    twelfth of its square: in all, less than a quarter more."""
    s, l = min(g.shape), max(g.shape)
    z = torch.linalg.svdvals(g.double().cpu())
    z = z / z.norm()
    p = z.clone()
    a, b, c = COEFS
    for _ in range(steps):
        p = a * p + b * p ** 3 + c * p ** 5
    return 1.25 * 2.0 ** -24 / math.sqrt(s * l) * (math.sqrt(s) + math.sqrt(l)) * float((p / z).norm() / p.norm())


def check(got, ref, steps, dtype, more=0.0):
    got = got.double().cpu()
    tol = tolerance(ref.shape, steps, dtype) + more
    assert bool(torch.isfinite(got).all())
    norm = float(ref.norm())
    assert float((got - ref).norm()) <= tol * norm, (float((got - ref).norm() / norm), tol)
    # and no element by itself: half a step, and eight times the rest's share of it
    rest = tol - torch.finfo(dtype).eps / 2
    worst = (got - ref).abs() - torch.finfo(dtype).eps / 2 * ref.abs()
    assert float(worst.max()) <= 8 * rest * norm / math.sqrt(ref.numel()) + 8 * rest * float(ref.abs().max()), float(worst.max())


def run(grads, outs, steps=5, dtype=F32, **kw):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.reserve_orthogonalize(dtype, [tuple(g.shape) if g.dim() == 2 else (1, g.numel()) for g in grads], steps)
    ctx.orthogonalize_batch([edgc.Tensor(g, o) for g, o in zip(grads, outs)], steps=steps, **kw)
    torch.cuda.synchronize()
    ctx.close()


def randn(shape, seed, dtype=F32, std=1e-3):
    return (std * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


SHAPES = [(1, 1), (1, 7), (7, 1), (5,), (5, 3), (3, 64), (64, 64), (65, 63), (63, 130), (128, 500), (500, 128), (129, 129), (300, 129), (333, 1000), (257, 256),
          (520, 520), (200, 2100), (2100, 200), (2, 5000), (4097, 65)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_matrix(shape, dtype):
    g = randn(shape, 1, dtype)
    out = torch.full_like(g, 9.0)
    run([g], [out], dtype=dtype)
    check(out, want(g, 5), 5, dtype)


@pytest.mark.parametrize("dtype, steps", [(F32, 5), (F32, 2), (BF16, 5), (BF16, 7), (BF16, 11)])
@pytest.mark.parametrize("shapes", [[(1000, 4000)], [(2100, 2333), (4100, 1999)], [(3001, 3001)]], ids=str)
def test_matrices_that_have_larger_tiles(shapes, dtype, steps):
    """Whole and shared tiles of 128 and 256 (smaller matrices have tiles of 64), into rows that are not aligned."""
    grads = [randn(s, 20 + i, dtype) for i, s in enumerate(shapes)]
    wide = [torch.full((m, n + 3), 6.0, dtype=dtype, device="cuda") for m, n in shapes]
    outs = [w[:, 1:1 + n] for w, (_, n) in zip(wide, shapes)]
    run(grads, outs, steps=steps, dtype=dtype)
    for g, o, w in zip(grads, outs, wide):
        check(o, want(g, steps, device="cuda").cpu(), steps, dtype)
        assert bool((w[:, 0] == 6.0).all()) and bool((w[:, -2:] == 6.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 11])
def test_numbers_of_steps(steps, dtype):
    grads = [randn((70, 200), 2, dtype), randn((200, 70), 3, dtype)]
    outs = [torch.empty_like(g) for g in grads]
    run(grads, outs, steps=steps, dtype=dtype)
    for g, o in zip(grads, outs):
        check(o, want(g, steps), steps, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_long_list_of_unlike_matrices_strided_with_scales(dtype):
    """More than are worked on together; rows further apart than they are long; some in place; what lies beside is not touched."""
    shapes = [(64, 64), (1, 9), (130, 70), (70, 130), (40, 300), (300, 40), (33, 33), (5, 5), (128, 128), (256, 64), (64, 320), (10, 100), (100, 10), (90, 91),
              (2, 2)] * 2
    host = [randn(s, 10 + i, dtype) for i, s in enumerate(shapes)]
    wide = [torch.full((m, n + 7), 5.0, dtype=dtype, device="cuda") for m, n in shapes]
    to = [torch.full((m, n + 3), 6.0, dtype=dtype, device="cuda") for m, n in shapes]
    grads = [w[:, 2:2 + n] for w, (_, n) in zip(wide, shapes)]
    for g, h in zip(grads, host):
        g.copy_(h)
    outs = [g if i % 3 == 0 else w[:, 1:1 + n] for i, (g, w, (_, n)) in enumerate(zip(grads, to, shapes))]
    scales = [0.5 + 0.25 * (i % 5) for i in range(len(shapes))]
    run(grads, outs, dtype=dtype, scales=scales)
    for i, (h, o, s) in enumerate(zip(host, outs, scales)):
        check(o, want(h, 5, s), 5, dtype)
        edge = wide[i] if i % 3 == 0 else to[i]
        lo, n = (2, shapes[i][1]) if i % 3 == 0 else (1, shapes[i][1])
        value = 5.0 if i % 3 == 0 else 6.0
        assert bool((edge[:, :lo] == value).all()) and bool((edge[:, lo + n:] == value).all())
        if i % 3:
            assert torch.equal(grads[i], h)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("std", [1e-30, 1e-18, 1.0, 1e18, 1e30])
def test_gradients_of_any_size(std, dtype):
    """Their squares pass the range of fp32 either way."""
    g = randn((96, 160), 5, dtype, std)
    out = torch.empty_like(g)
    run([g], [out], dtype=dtype, eps=0.0)
    check(out, want(g, 5, eps=0.0), 5, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_eps_beside_a_small_norm(dtype):
    g = randn((96, 160), 6, dtype, 1e-6)
    out = torch.empty_like(g)
    run([g], [out], dtype=dtype, eps=1e-3)
    check(out, want(g, 5, eps=1e-3), 5, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_and_what_is_not_finite(dtype):
    """Zeros stay zeros; Inf or NaN makes its own matrix NaN, whole, and no other."""
    grads = [torch.zeros(80, 100, dtype=dtype, device="cuda"), randn((80, 100), 7, dtype), randn((80, 100), 8, dtype), randn((100, 80), 9, dtype),
             torch.zeros(1, 5, dtype=dtype, device="cuda")]
    grads[1][3, 4] = float("inf")
    grads[3][99, 79] = float("nan")
    outs = [torch.full_like(g, 2.0) for g in grads]
    run(grads, outs, dtype=dtype, eps=0.0)
    assert bool((outs[0] == 0).all()) and bool((outs[4] == 0).all())
    assert bool(torch.isnan(outs[1]).all()) and bool(torch.isnan(outs[3]).all())
    check(outs[2], want(grads[2], 5, eps=0.0), 5, dtype)


def test_a_few_strong_directions_above_noise():
    """Singular values over four decades, as gradients have them: the smallest come out as accurately as the rest of the matrix."""
    u, v = randn((256, 8), 20, std=1.0), randn((512, 8), 21, std=1.0)
    g = (u * 0.3 ** torch.arange(8, device="cuda")) @ v.t() + randn((256, 512), 22, std=1e-3)
    out = torch.empty_like(g)
    run([g], [out])
    check(out, want(g, 5), 5, F32, of_the_input(g, 5))


@pytest.mark.parametrize("coefs", [(1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375), (0.5, 0.5, 0.0)])
def test_other_coefficients(coefs):
    grads = [randn((70, 200), 2), randn((200, 70), 3)]
    outs = [torch.empty_like(g) for g in grads]
    run(grads, outs, coefficients=coefs)
    for g, o in zip(grads, outs):
        check(o, want(g, 5, coefs=coefs), 5, F32)


def test_the_same_list_gives_the_same_bits_also_from_a_graph():
    shapes = [(200, 300), (300, 200), (65, 64)]
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.reserve_orthogonalize(F32, shapes)
    grads, outs = [torch.zeros(s, device="cuda") for s in shapes], [torch.empty(s, device="cuda") for s in shapes]
    batch = edgc.PreparedBatch([edgc.Tensor(g, o) for g, o in zip(grads, outs)])
    fill = lambda seed: [g.copy_(randn(g.shape, seed + i)) for i, g in enumerate(grads)]
    side = torch.cuda.Stream()
    fill(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.orthogonalize_batch(batch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.orthogonalize_batch(batch)
    for seed in (1, 5, 9, 1):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outs]
        ctx.orthogonalize_batch(batch)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))
        check(outs[0], want(grads[0], 5), 5, F32)
    ctx.close()


def test_refusals():
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    g = torch.zeros(40, 50, device="cuda")
    t = [edgc.Tensor(g, g)]

    def refused(match, f, *a, **kw):
        with pytest.raises(edgc.EdgcError, match=match) as e:
            f(*a, **kw)
        assert e.value.code == -1
    refused("reserve_orthogonalize", ctx.orthogonalize_batch, t)                # nothing reserved
    ctx.reserve_orthogonalize(F32, [(40, 50)])
    ctx.orthogonalize_batch(t)
    ctx.orthogonalize_batch([edgc.Tensor(g, torch.empty_like(g)) for _ in range(3)])    # one after the other in the same scratch
    ctx.orthogonalize_batch([])
    refused("reserve_orthogonalize", ctx.orthogonalize_batch, [edgc.Tensor(torch.zeros(40, 500, device="cuda"), torch.zeros(40, 500, device="cuda"))])
    for steps in (0, 65):
        refused("steps", ctx.orthogonalize_batch, t, steps=steps)
        refused("steps", ctx.reserve_orthogonalize, F32, [(4, 4)], steps)
    ctx.reserve_orthogonalize(F32, [(40, 50)], steps=3)
    refused("larger than", ctx.orthogonalize_batch, t)                          # a second X
    for eps in (-1.0, math.nan, math.inf):
        refused("eps", ctx.orthogonalize_batch, t, eps=eps)
    for coefs in ((math.nan, 0, 0), (3.4445, math.inf, 1.0), (100.0, 0.0, 0.0), (1.0, 0.0, 50.0)):
        refused("coefficients", ctx.orthogonalize_batch, t, coefficients=coefs)
    refused("scales", ctx.orthogonalize_batch, t, scales=[math.inf])
    with pytest.raises(ValueError):
        ctx.orthogonalize_batch(t, scales=[1.0, 1.0])
    refused("side", ctx.reserve_orthogonalize, F32, [(2 ** 14 + 1, 2 ** 14 + 1)])
    refused("side", ctx.reserve_orthogonalize, F32, [(4, 2 ** 20 + 1)])
    refused("empty", ctx.reserve_orthogonalize, F32, [(0, 4)])
    refused("null gradient", ctx.orthogonalize_batch, [edgc.Tensor(g, None)])
    ctx.reserve_orthogonalize(F32, [])
    refused("reserve_orthogonalize", ctx.orthogonalize_batch, t)
    ctx.close()

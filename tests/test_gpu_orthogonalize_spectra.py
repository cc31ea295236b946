"""The orthogonalised update of gradients whose singular values lie far apart, as those of few directions above noise do: what A loses of the small ones is
carried on by every further step on it."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

COEFS = (3.4445, -4.7750, 2.0315)
F32, BF16 = torch.float32, torch.bfloat16


def steps_of(g, steps, coefs=COEFS, dtype=torch.float64, eps=1e-7):
    """The steps on the matrix itself, s x l with s <= l, in `dtype`."""
    a, b, c = coefs
    x = g.double()
    x = (x / (x.norm() + eps)).to(dtype)
    for _ in range(steps):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def gradient(kind, s, l):
    if kind == "one above noise":
        return randn((s, 1), 1) @ randn((1, l), 2) + 1e-3 * randn((s, l), 3)
    if kind == "eight above noise":
        return (randn((s, 8), 1) * 0.3 ** torch.arange(8, dtype=torch.float64)) @ randn((8, l), 2) + 1e-3 * randn((s, l), 3)
    if kind == "one, rounded":                              # (bf16's own roundings are the other directions)
        return randn((s, 1), 1) @ randn((1, l), 2)
    if kind == "many above noise":
        return (randn((s, 32), 1) * 0.8 ** torch.arange(32, dtype=torch.float64)) @ randn((32, l), 2) + randn((s, l), 3)
    u, v = torch.linalg.qr(randn((s, s), 1))[0], torch.linalg.qr(randn((l, s), 2))[0]
    return (u * 10.0 ** (-4 * torch.linspace(0, 1, s, dtype=torch.float64))) @ v.t()       # evenly over four decades


def run(g, steps, coefs=COEFS, reserved=None):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.reserve_orthogonalize(g.dtype, [tuple(g.shape)], reserved or steps)
    out = torch.full_like(g, 9.0)
    ctx.orthogonalize_batch([edgc.Tensor(g, out)], steps=steps, coefficients=coefs)
    torch.cuda.synchronize()
    ctx.close()
    return out


@pytest.mark.parametrize("steps", [5, 4, 3])
@pytest.mark.parametrize("kind", ["one above noise", "eight above noise", "one, rounded", "four decades"])
@pytest.mark.parametrize("s, l", [(16, 2048), (64, 4096), (16, 65536), (256, 2048), (512, 16384), (1024, 16384)])
def test_bf16_updates_are_off_by_little_more_than_their_rounding(s, l, kind, steps):
    """What is wrong with W is wrong with all of a row in the same way: it lies in the s directions of l that the update has, of which roundings, each its own,
    have sqrt(s / l).  They are at most half a step, evenly spread: 2^-8 / sqrt 3 in the norm; a quarter more for what 256 directions and more wander by.
    The rest: an A_0 off by d of its largest value, 2^-23 of the planes and 2^-25 sqrt l of sums of l products; as a matrix of such errors 2 / sqrt s of it in the
    norm; |b| / a = 1.4 of that in W; twelve times more in each further step on the same A: two of them, and of a second A one.  And sqrt(3 l) 2^-25 of each of
    ten products of X."""
    g = gradient(kind, s, l).to(BF16).cuda()
    want = steps_of(g, steps)
    err = run(g, steps).double() - want
    assert bool(torch.isfinite(err).all())
    inside = err.cpu() @ torch.linalg.qr(want.t().cpu())[0]
    d = 2.0 ** -23 + math.sqrt(l) * 2.0 ** -25
    rounding = 1.25 * math.sqrt(s / l) * 2.0 ** -8 / math.sqrt(3)
    bound = rounding + 1.4 * (1 + 12 + 144 + 1 + 12) * min(1.0, 2 / math.sqrt(s)) * d + 10 * math.sqrt(3 * l) * 2.0 ** -25
    off = float(inside.norm()) / float(want.norm())
    print(f"{s}x{l} {kind}, {steps} steps: {off:.2e} of {bound:.2e}")
    assert off <= bound, (off, bound)


@pytest.mark.parametrize("steps", [5, 3, 4, 6, 7, 8])
@pytest.mark.parametrize("kind", ["four decades", "eight above noise", "one above noise"])
@pytest.mark.parametrize("s, l", [(64, 64), (512, 512), (200, 1000), (16, 32768)])
def test_fp32_updates_are_off_by_a_few_times_what_fp32_products_are(s, l, kind, steps):
    """Beside the same steps on X itself in fp32.  The planes' roundings are twice those of fp32, and a step on the same A, not on X, as large again: four times
    in all."""
    g = gradient(kind, s, l).float()
    want = steps_of(g, steps)
    rel = lambda x: float((x.double().cpu() - want).norm() / want.norm())
    plain, off = rel(steps_of(g, steps, dtype=F32)), rel(run(g.cuda(), steps))
    print(f"{s}x{l} {kind}, {steps} steps: {off:.2e}, fp32 products {plain:.2e}")
    assert off <= 4 * plain, (off, plain)


@pytest.mark.parametrize("steps", [5, 3, 6])
@pytest.mark.parametrize("s, l", [(62, 192), (64, 98), (64, 1152), (128, 512), (250, 250), (512, 2048)])
def test_fp32_updates_of_many_directions_above_noise(s, l, steps):
    """Where no direction is far below the others, fp32 products are off by little, and two steps on the same A by no more than twice that; and both operands of the
    last product, Q and X, are rounded to 22 bits and the residual's sign, 2^-23 of it each, which fp32 operands are not."""
    g = gradient("many above noise", s, l).float()
    want = steps_of(g, steps)
    rel = lambda x: float((x.double().cpu() - want).norm() / want.norm())
    plain, off = rel(steps_of(g, steps, dtype=F32)), rel(run(g.cuda(), steps))
    print(f"{s}x{l} many above noise, {steps} steps: {off:.2e}, fp32 products {plain:.2e}")
    assert off <= 2 * plain + 2.0 ** -22, (off, plain)


@pytest.mark.parametrize("steps", [3, 2, 5])
@pytest.mark.parametrize("coefs", [(5.0, -20.0, 16.0), (-5.0, 20.0, -16.0), (4.1, -7.4, 3.25)])
def test_coefficients_that_carry_errors_further(coefs, steps):
    """a^2 = 25 or 17 in every further step on the same A."""
    g = gradient("eight above noise", 64, 300).float()
    want = steps_of(g, steps, coefs)
    rel = lambda x: float((x.double().cpu() - want).norm() / want.norm())
    plain, off = rel(steps_of(g, steps, coefs, dtype=F32)), rel(run(g.cuda(), steps, coefs, reserved=5))
    print(f"{coefs}, {steps} steps: {off:.2e}, fp32 products {plain:.2e}")
    assert off <= 8 * plain, (off, plain)


@pytest.mark.parametrize("kind", ["one above noise", "four decades"])
def test_large_matrices(kind):
    """Tiles of 128."""
    g = gradient(kind, 1500, 3000).float()
    want = steps_of(g, 5)
    rel = lambda x: float((x.double().cpu() - want).norm() / want.norm())
    plain, off = rel(steps_of(g, 5, dtype=F32)), rel(run(g.cuda(), 5))
    print(f"{kind}: {off:.2e}, fp32 products {plain:.2e}")
    assert off <= 4 * plain, (off, plain)


def test_a_reservation_for_few_steps_is_for_few_and_one_for_more_for_any():
    g = gradient("eight above noise", 40, 60)
    for dtype, few in ((F32, 3), (BF16, 5)):
        x = g.to(dtype).cuda()
        for steps in (1, few):
            run(x, steps, reserved=1)
        with pytest.raises(edgc.EdgcError, match="larger than"):
            run(x, few + 1, reserved=few)
        out = run(x, 64, reserved=few + 1)
        assert bool(torch.isfinite(out).all())
    # coefficients for which X is formed again in fewer steps need nothing else
    x = g.float().cuda()
    want = steps_of(g.float(), 3, (5.0, -20.0, 16.0))
    assert float((run(x, 3, (5.0, -20.0, 16.0)).double().cpu() - want).norm()) < 1e-3 * float(want.norm())

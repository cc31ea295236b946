"""The orthogonalised update where its scale, or the eps beside the norm, takes it far from one."""
import math

import pytest
import torch

import paper_2511_10333_amd as edgc

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
F32, BF16 = torch.float32, torch.bfloat16


def want(g, steps, scale, eps):
    x = g.double().cpu()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        gram = x @ x.t()
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    return scale * (x.t() if tall else x)


def run(g, steps, scale=1.0, eps=1e-7):
    ctx = edgc.Context(0, max_bins=64, max_rank=4, max_rows=64, max_cols=64)
    ctx.reserve_orthogonalize(g.dtype, [tuple(g.shape)], steps)
    out = torch.full_like(g, 9.0)
    ctx.orthogonalize_batch([edgc.Tensor(g, out)], steps=steps, eps=eps, scales=[scale])
    torch.cuda.synchronize()
    ctx.close()
    return out


def check(got, ref):
    """Matrices of normally distributed elements, whose singular values are alike: as 22 bits of an operand and fp32 sums allow after five steps and more, 1e-5
    in the norm (the planes' 2^-23 twelve times larger in each of two steps, 2 / sqrt s of it), and half a step of the type; and the spacing of the smallest
    numbers of an fp32."""
    eps = torch.finfo(got.dtype).eps / 2
    err, norm = (got.double().cpu() - ref).norm(), ref.norm()
    floor = math.sqrt(ref.numel()) * 2.0 ** (-150 if got.dtype is F32 else -134)
    assert bool(torch.isfinite(got).all())
    assert float(err) <= (1e-5 + eps) * float(norm) + floor, (float(err / norm), float(norm))


def randn(shape, std, dtype, seed=3):
    return (std * torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", [2, 5])
@pytest.mark.parametrize("scale", [1e37, -1e30, 1e-25, -1e-30, 1e-35, 1e-37])
def test_scales(scale, steps, dtype):
    for shape in ((96, 160), (160, 96)):
        g = randn(shape, 1e-3, dtype)
        check(run(g, steps, scale), want(g, steps, scale, 1e-7))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", [1, 3, 5, 7])
@pytest.mark.parametrize("std, eps", [(1e-5, 1e-2), (1e-10, 1e-3), (1e-16, 1e-7), (1e-22, 1e-7), (1e-3, 1e25), (1e-30, 1e-7)])
def test_an_eps_far_above_the_norm(std, eps, steps, dtype):
    g = randn((96, 160), std, dtype)
    check(run(g, steps, eps=eps), want(g, steps, 1.0, eps))

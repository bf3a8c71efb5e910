"""Norms of rows so small, with an eps so small, that the mean of their squares is below the smallest normal float.

Tolerance: squares and their sum are rounded to multiples of 2^-149, and the rows' means are at least 2^-131: a square is off by 2^-19 of the mean, the mean of
many by less, its root by half of that: with the 2^-18 of other rows 2^-17 of a value; gradients, whose terms hold the root's reciprocal three times, 2^-16 of
the terms' sum, and the rounding to the type."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-39, 1e-37])
@pytest.mark.parametrize("D,pairs", [(64, 0), (128, 64), (72, 36), (7, 3), (512, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_rows(dtype, D, pairs, eps):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D)
    q = torch.randn((40, 3, D), generator=gen, device="cuda")
    size = torch.tensor([3e-20, 1e-19, 3e-19, 1.0], device="cuda").repeat(10)
    q = (q / q.square().mean(-1, keepdim=True).sqrt() * size[:, None, None]).to(dtype)
    g = torch.randn((40, 3, D), generator=gen, device="cuda").to(dtype)
    frequency, axis = pkg.axis_frequencies((pairs,))
    positions = torch.zeros((1, 40), dtype=torch.int32, device="cuda")         # (not turned: the norm alone)
    x, h = q.double(), g.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + torch.tensor(eps, dtype=torch.float32).double().item())
    y = pkg.norm_rotate(q, None, None, None, positions, frequency, axis, eps=eps)[0].double()
    assert bool(((y - x * r).abs() <= (HALF_UNIT[dtype] + 2.0 ** -17) * (x * r).abs()).all())
    w = torch.ones(D, device="cuda")
    dx, _, dw, _ = pkg.norm_rotate_backward(g, None, q, None, w, None, positions, frequency, axis, eps=eps)
    want = r * (h - x * r * r * (h * x).mean(-1, keepdim=True))
    terms = r * (h.abs() + x.abs() * r * r * (h * x).abs().mean(-1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= HALF_UNIT[dtype] * want.abs() + 2.0 ** -16 * terms).all())
    assert bool(((dw.double() - (h * x * r).sum((0, 1))).abs() <= 2.0 ** -15 * (h * x * r).abs().sum((0, 1))).all())


def test_rows_of_zeros_with_the_smallest_eps():
    q = torch.zeros((5, 2, 32), device="cuda")
    frequency, axis = pkg.axis_frequencies((16,))
    positions = torch.arange(5, device="cuda")[None]
    g = torch.ones_like(q)
    for eps in (1e-45, 1e-42, 1e-38):
        assert not pkg.norm_rotate(q, None, None, None, positions, frequency, axis, eps=eps)[0].any()
        dx = pkg.norm_rotate_backward(g, None, q, None, None, None, torch.zeros_like(positions), frequency, axis, eps=eps)[0]
        want = torch.tensor(eps, dtype=torch.float32).double().item() ** -0.5
        assert bool(((dx.double() - want).abs() <= 2.0 ** -17 * want).all())

"""Gradients of group norm over large pictures of which there are many: how many pixels a thread adds up one after another is bounded.

With n equal terms t a running sum in 32 bits is off by half a unit of each of its values at most, 2^-24 (n / 2) of n t: with n = 512 by 2^-16.  Products add 2^-24 to that, sums over lanes and channels
less than 2^8 roundings, 2^-16; over chunks they are made in 64 bits: 2^-15 in all.  (A running sum of 8192 terms of 0.9 is off by 2^-13.7, of 0.1 by 2^-13.9, in the same direction every time.)"""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images,pixels,C,G", [(512, 8192, 129, 1), (1, 2 ** 22 + 5, 129, 3)])
@pytest.mark.parametrize("g,u", [(0.9, 0.7), (0.1, 1.0)])
def test_sums_of_equal_terms(images, pixels, C, G, g, u):
    x = torch.full((images, pixels, C), u, device="cuda")
    grad = torch.full_like(x, g)
    stats = torch.tensor([0.0, 1.0], device="cuda").expand(images, G, 2).contiguous()          # (u = x: what forward gives has a part in the formulas only)
    w, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    dx, dw, db = pkg.group_norm_backward(grad, x, G, w, b, stats)
    g, u = float(grad[0, 0, 0]), float(x[0, 0, 0])
    n = images * pixels
    assert bool(((db.double() - n * g).abs() <= 2.0 ** -15 * n * g).all()), float((db.double() / (n * g) - 1).abs().max())
    assert bool(((dw.double() - n * g * u).abs() <= 2.0 ** -15 * n * g * u).all()), float((dw.double() / (n * g * u) - 1).abs().max())
    # dx = g - mean g - u mean g u = - u g u: the means as their sums, and three roundings
    assert bool(((dx + g * u * u).abs() <= 2.0 ** -15 * (2 * g + 2 * g * u * u)).all())

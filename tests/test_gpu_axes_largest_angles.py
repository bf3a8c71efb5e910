"""Angles up to the largest floats, sine and cosine against the C library's in 64 bits (which reduces them exactly): 2^-21 of |x| + |y|, as for other angles."""
import math

import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu


def test_angles_up_to_the_largest_floats():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    exponents = torch.arange(0, 127).repeat_interleave(2)
    pairs = 254
    frequency = ((1 + torch.rand(pairs, generator=gen, device="cuda")) * 2.0 ** exponents.to("cuda", torch.float32)).clamp(max=torch.finfo(torch.float32).max)
    frequency[253] = torch.finfo(torch.float32).max
    axis = torch.zeros(pairs, dtype=torch.int32, device="cuda")
    positions = torch.tensor([[1, -1]], device="cuda")
    q = torch.randn((2, 3, 508), generator=gen, device="cuda")
    got = pkg.rotate_axes(q, None, positions, frequency, axis)[0].double().cpu()
    x, angles = q.double().cpu(), frequency.double().tolist()
    c, s = (torch.tensor([f(v) for v in angles], dtype=torch.float64) for f in (math.cos, math.sin))
    for token, sign in ((0, 1.0), (1, -1.0)):
        u, v = x[token, :, :pairs], x[token, :, pairs:]
        want = torch.cat([u * c - sign * v * s, sign * u * s + v * c], -1)
        slack = 2.0 ** -24 * want.abs() + 2.0 ** -21 * (u.abs() + v.abs()).repeat(1, 2)
        off = (got[token] - want).abs() - slack
        assert bool((off <= 0).all()), [(math.log2(angles[j % pairs]), float(off[:, j].max())) for j in range(2 * pairs) if float(off[:, j].max()) > 0][:8]

"""Group norm of pictures whose groups hold one value each, or values very close to each other and far from 0: what 1 / sqrt(eps) would make of an error of the mean.

A sum of n equal values v of 24 bits, n below 2^29, is exact in 64 bits, and so is its quotient by n once it is rounded to 32: the mean is v, the squares are 0, y is the bias."""
import pytest
import torch

import paper_1911_00472_amd as pkg
import test_gpu_group_norm as norm

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [  # x, groups: one pass by 256 threads and by 512, runs of every length; several pictures to a workgroup; two passes, wide ones, chunks joined by their own launch
    ((1, 9, 9, 8), 2), ((3, 7, 7, 45), 3), ((2, 5, 23, 12), 3), ((1, 13, 13, 64), 1), ((2, 28, 28, 128), 32), ((4, 30, 30, 64), 2), ((1, 3, 1000), 8), ((2, 1, 1, 6), 2),
    ((2100, 3, 1, 12), 2), ((5000, 1, 1, 1000), 8), ((2100, 7, 1, 40), 5), ((100001, 3, 3), 1),
    ((2, 150, 149, 32), 8), ((1, 40, 2304), 32), ((5, 37, 53, 90), 6), ((1, 301, 299, 24), 24), ((1, 257, 255, 6), 1),
]


@pytest.mark.parametrize("dtype", norm.TYPES)
@pytest.mark.parametrize("shape,G", SHAPES)
def test_equal_values(shape, G, dtype):
    gen = norm.generator(G)
    for v in (900.1, -0.1, 3.3e4, 1e-3):
        # each group of each picture its own value
        of_group = (v * (1 + torch.rand((shape[0],) + (1,) * (len(shape) - 2) + (G,), generator=gen, device="cuda"))).clamp(-6e4, 6e4).to(dtype)
        x = of_group.repeat_interleave(shape[-1] // G, -1).expand(shape).contiguous()
        b = torch.randn(shape[-1], generator=gen, device="cuda").to(dtype)
        y, stats = pkg.group_norm_forward(x, G, None, b, EPS)
        assert torch.equal(stats[..., 0], of_group.float().view(shape[0], G)), v
        assert bool(((stats[..., 1] - EPS ** -0.5).abs() <= 2.0 ** -22 * EPS ** -0.5).all())
        assert torch.equal(y, b.expand(shape)), v


@pytest.mark.parametrize("shape,G", SHAPES[2:])
def test_values_next_to_each_other(shape, G):
    """900 and the float behind it, 2^-14 away, by chance.  Roundings keep the order of numbers, sums of up to 2^28 such values are exact in 64 bits: every mean, of a thread or of a group, lies between the two,
    and so is off by 2^-14 at most, as x - m is; r is 1 / sqrt(eps) at most and a unit or two."""
    x = 900 + 2.0 ** -14 * torch.randint(0, 2, shape, generator=norm.generator(1), device="cuda").float()
    y, stats = pkg.group_norm_forward(x, G, eps=EPS)
    m = norm.grouped(x, G).mean((1, 3))
    assert bool(((stats[..., 0].double().cpu() - m).abs() <= 2.0 ** -14).all())
    assert bool((y.abs() <= 2.0 ** -14 * EPS ** -0.5 * (1 + 2.0 ** -20)).all())

"""Angles that are not numbers: a frequency of NaN or infinity, and a product that overflows, make NaN of the pairs they turn and of nothing else."""
import math

import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_only_the_pairs_of_the_angle_are_nan(dtype, adjacent):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    q = torch.randn((3, 9, 5, 40), generator=gen, device="cuda").to(dtype)
    frequency, axis = pkg.axis_frequencies((8, 8))
    positions = torch.randint(1, 50, (2, 3, 9), generator=gen, device="cuda")
    positions[0, 1, 4], positions[1, 2, 7] = 0, 2 ** 40
    bad = frequency.clone()
    bad[1], bad[5], bad[11], bad[13] = math.nan, math.inf, 3e30, -math.inf             # 0 inf is NaN; 2^40 3e30 is infinite
    nan = torch.zeros((3, 9, 40), dtype=torch.bool)
    for j, where in ((1, torch.ones((3, 9), dtype=torch.bool)), (5, torch.ones((3, 9), dtype=torch.bool)), (11, positions[1].cpu() == 2 ** 40), (13, torch.ones((3, 9), dtype=torch.bool))):
        for e in ((2 * j, 2 * j + 1) if adjacent else (j, j + 16)):
            nan[..., e] = where
    nan = nan[:, :, None].expand(3, 9, 5, 40)
    for inverse in (False, True):
        got = pkg.rotate_axes(q, None, positions, bad, axis, adjacent=adjacent, inverse=inverse)[0].cpu()
        clean = pkg.rotate_axes(q, None, positions, frequency, axis, adjacent=adjacent, inverse=inverse)[0].cpu()
        assert torch.equal(torch.isnan(got), nan)
        same = ~nan
        for e in ((22, 23) if adjacent else (11, 27)):         # (the pair of another frequency)
            same[..., e] = False
        assert torch.equal(got[same], clean[same])
    w = torch.ones(40, device="cuda")
    got = pkg.norm_rotate(q, None, w, None, positions, bad, axis, adjacent=adjacent)[0].cpu()
    assert torch.equal(torch.isnan(got), nan)

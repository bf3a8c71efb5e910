"""Group norm of thousands of small pictures whose runs of channels do not divide a workgroup's threads: no pixel of a picture is left out, of its statistics or of what is written."""
import numpy as np
import pytest
import torch

import paper_1911_00472_amd as pkg
import test_gpu_group_norm as norm

pytestmark = pytest.mark.gpu
EPS = 1e-5

# pixels, channels, groups: at the border of what two runs of fewer than 16 bytes in each of 256 threads hold, and behind it
PICTURES = [(3, 300, 4), (5, 180, 6), (7, 140, 7), (9, 108, 4), (9, 53, 1), (11, 90, 6), (17, 60, 4), (5, 202, 2), (73, 7, 1), (5, 198, 3)]


@pytest.mark.parametrize("dtype", norm.TYPES)
@pytest.mark.parametrize("images", [2048, 4099])
@pytest.mark.parametrize("pixels,C,G", [(p + more, C, G) for p, C, G in PICTURES for more in (-1, 0, 1)])
def test_small_pictures_are_held_whole(pixels, C, G, images, dtype):
    gen = norm.generator(images + C + pixels)
    x = norm.make((images, pixels, C), dtype, gen)
    w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
    kind = norm.ACTIVATIONS[(pixels + C) % 4]
    out = torch.full_like(x, float("nan"))                     # (what is not written shows)
    y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind, out=out)
    norm.check_forward(x, G, w, b, EPS, kind, y, stats)
    g = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
    dx = torch.full_like(x, float("nan"))
    norm.check_backward(g, x, G, w, b, stats, kind, *pkg.group_norm_backward(g, x, G, w, b, stats, kind, dx=dx))


@pytest.mark.parametrize("seed", range(16))
def test_small_pictures_drawn_by_chance(seed):
    rng = np.random.default_rng(500 + seed)
    for _ in range(4):
        C = int(2 ** rng.uniform(0, 10.5))
        G = int(rng.choice([g for g in range(1, min(C, 64) + 1) if C % g == 0]))
        pixels = int(max(1, min(2 ** rng.uniform(0, 7), 1200 / C)))
        images = int(min(rng.integers(2048, 20000), 6e6 // (C * pixels)))
        dtype, kind, pad = norm.TYPES[rng.integers(3)], norm.ACTIVATIONS[rng.integers(4)], int(rng.integers(0, 5)) if rng.random() < 0.3 else 0
        print(images, pixels, C, G, dtype, kind, pad, flush=True)
        gen = norm.generator(seed)
        x, out, dx = (norm.make((images, pixels, C + pad), dtype, gen)[..., pad:] for _ in range(3))
        w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
        y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind, out=out.fill_(float("nan")))
        norm.check_forward(x, G, w, b, EPS, kind, y, stats)
        g = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
        norm.check_backward(g, x, G, w, b, stats, kind, *pkg.group_norm_backward(g, x, G, w, b, stats, kind, dx=dx.fill_(float("nan"))))

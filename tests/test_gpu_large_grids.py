"""Calls of more work items than one launch holds (2^32): the smallest of each kind, many rows of a few elements each.

Tolerances: those of the operators' other tests.  Rotation: 2^-21 of |x| + |y| and the rounding to the type; the loss: 2^-17 of its parts and 2^-22 of its
terms (below 32 here), the gradient 2^-16 of its terms and the rounding; patch rows: 2^-22 of the largest factor and the rounding."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
BFLOAT = 2.0 ** -8


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def test_many_rows_of_a_few_classes():
    """2^26 rows of a wavefront each."""
    N, V, T, a, b = 2 ** 26 + 5, 3, 2.0, 0.6, 0.4
    gen = generator(1)
    z = torch.randn((N, V), generator=gen, device="cuda").bfloat16()
    index = torch.randint(0, V, (N, 1), generator=gen, device="cuda", dtype=torch.int32)
    t = torch.randn((N, 1), generator=gen, device="cuda").bfloat16()
    labels = torch.randint(0, V, (N,), generator=gen, device="cuda")
    weight = torch.rand(N, generator=gen, device="cuda") + 0.25
    how = dict(labels=labels, temperature=T, distill_part=a, label_part=b)
    loss, sums = pkg.distill_forward(z, index, t, **how)
    back = pkg.distill_backward(weight, z, index, t, sums, **how)
    both, step = pkg.distill_step(z, index, t, weight, **how)
    for i in range(0, N, 2 ** 24):                             # (a single entry: all of the teacher's weight is on it)
        rows = slice(i, i + 2 ** 24)
        x, at, label = z[rows].double(), index[rows].long(), labels[rows, None]
        by_t, by_one = torch.log_softmax(x / T, 1), torch.log_softmax(x, 1)
        want = -(a * T * T * by_t.gather(1, at) + b * by_one.gather(1, label))[:, 0]
        w = weight[rows].double()
        slack = 2.0 ** -17 * (a * T * T + b) + 2.0 ** -17
        assert bool(((loss[rows] - want).abs() <= slack).all()) and bool(((both[rows] - want * w).abs() <= slack * w).all()), i
        one = torch.zeros_like(x).scatter_(1, at, a * T).scatter_add_(1, label, torch.full_like(label, b, dtype=torch.float64))
        dense = a * T * by_t.exp() + b * by_one.exp()
        grad, size = (dense - one) * w[:, None], (dense + one) * w[:, None]
        for got in (back, step):
            assert bool(((got[rows].double() - grad).abs() <= BFLOAT * grad.abs() + 2.0 ** -16 * size + 2.0 ** -125).all()), i


def test_many_sequences_of_two_tokens():
    """2^24 sequences that do not lie behind each other: a workgroup each."""
    B, T, H, D = 2 ** 24 + 3, 2, 2, 2
    gen = generator(2)
    q = torch.randn((B, H, T, D), generator=gen, device="cuda").bfloat16().transpose(1, 2)
    positions = torch.randint(0, 100, (1, B, T), generator=gen, device="cuda", dtype=torch.int32)
    frequency, axis = torch.tensor([0.37], device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pkg.rotate_axes(q, None, positions, frequency, axis)[0]
    for i in range(0, B, 2 ** 22):
        rows = slice(i, i + 2 ** 22)
        x = q[rows].double()
        angle = (positions[0, rows].float() * frequency).double()[..., None]
        c, s = torch.cos(angle), torch.sin(angle)
        want = torch.stack([x[..., 0] * c - x[..., 1] * s, x[..., 0] * s + x[..., 1] * c], -1)
        slack = BFLOAT * want.abs() + 2.0 ** -21 * x.abs().sum(-1, keepdim=True) + 2.0 ** -126
        assert bool(((got[rows].double() - want).abs() <= slack).all()), i


def test_many_patches_of_a_pixel():
    """2^30 rows, 64 to a workgroup."""
    H, W = 1073743, 1000
    pixels = torch.randint(0, 256, (H * W,), generator=generator(3), device="cuda", dtype=torch.uint8)
    shapes, offsets, first, rows = pkg.patch_layout([(H, W)], 1, 1)
    assert rows > 64 * (2 ** 32 // 256)
    got, positions = pkg.patch_rows(pixels, shapes, offsets, first, rows, 1, (0.45,), (4.0,))
    lines = 65536
    for y in range(0, H, lines):
        part = slice(y * W, min(y + lines, H) * W)
        want = (pixels[part].double() / 255 - 0.45) * 4.0
        assert bool(((got[part, 0].double() - want).abs() <= BFLOAT * want.abs() + 2.0 ** -20).all()), y
        n = want.numel() // W
        assert not positions[0, part].any()
        assert bool((positions[1, part].view(n, W) == torch.arange(y, y + n, dtype=torch.int32, device="cuda")[:, None]).all()), y
        assert bool((positions[2, part].view(n, W) == torch.arange(W, dtype=torch.int32, device="cuda")).all()), y

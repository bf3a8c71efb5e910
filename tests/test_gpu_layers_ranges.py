"""Group norm, position bias and dropout over wide ranges: of numbers, of pictures, of elements behind 2^32, of shapes drawn by chance."""
import numpy as np
import pytest
import torch

import paper_1911_00472_amd as pkg
import test_gpu_dropout as drop
import test_gpu_group_norm as norm
import test_gpu_position_bias as places

pytestmark = pytest.mark.gpu
EPS = 1e-5


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def check_pairs(x, y, dx, dw):
    """Pictures of one or two pixels, a group to each channel: u = (x - m) r, and the gradient x of y times 1."""
    images, pixels = x.shape[:2]
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[x.dtype]
    total = torch.zeros(x.shape[2], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    step = max(1, 2 ** 23 // x.shape[2])
    for i in range(0, images, step):
        v = x[i:i + step].double()
        m = v.mean(1, keepdim=True)
        r = ((v - m).square().mean(1, keepdim=True) + EPS) ** -0.5
        u = (v - m) * r
        # (m to 2^-23 of the larger value, which is below 2^3: u to 2^-20 r)
        assert bool(((y[i:i + step].double() - u).abs() <= half * u.abs() + 2.0 ** -20 * r + 2.0 ** -20).all()), i
        total += (v * u).sum((0, 1))
        size += (v * u).abs().sum((0, 1)) + 2.0 ** -6 * (v.abs() * r).sum((0, 1))
        want = r * (v - m - u * (v * u).mean(1, keepdim=True))
        assert bool(((dx[i:i + step].double() - want).abs() <= half * want.abs() + 2.0 ** -14 * r * (v.abs() + v.abs().mean(1, keepdim=True)) * (1 + 2.0 ** -4 * r) + 2.0 ** -100).all()), i
    assert bool(((dw.double() - total).abs() <= 2.0 ** -12 * size).all())


@pytest.mark.parametrize("pixels,images", [(2, 2 ** 24 + 8), (1, 2 ** 24 + 3)])
def test_millions_of_small_pictures(pixels, images):
    """Hundreds of them to a workgroup, the last of them not full."""
    x = torch.randn((images, pixels, 2), generator=generator(1), device="cuda").bfloat16()
    y, stats = pkg.group_norm_forward(x, 2)
    dx, dw, _ = pkg.group_norm_backward(x, x, 2, torch.ones(2, device="cuda"), None, stats)
    check_pairs(x, y, dx, dw)


def test_more_workgroups_than_a_launch_has():
    """2^24 workgroups of 256 threads and 128 more: pictures of two pixels of 4096 channels, 32 channels to a workgroup."""
    x = torch.randn((2 ** 17 + 1, 2, 4096), generator=generator(8), device="cuda")
    y, stats = pkg.group_norm_forward(x, 4096)
    dx, dw, _ = pkg.group_norm_backward(x, x, 4096, torch.ones(4096, device="cuda"), None, stats)
    check_pairs(x, y, dx, dw)


@pytest.mark.parametrize("dtype", norm.TYPES)
@pytest.mark.parametrize("images", [2047, 2048, 4095, 4096, 8193, 40001])
@pytest.mark.parametrize("pixels,C,G", [(1, 8, 1), (1, 1, 1), (1, 24, 3), (4, 32, 4), (1, 1024, 1), (1, 520, 65), (3, 12, 2), (2, 6, 3), (7, 40, 5), (9, 16, 16), (1, 2000, 10), (5, 3, 1), (2, 90, 9)])
def test_many_small_pictures(pixels, C, G, images, dtype):
    """Several pictures of a workgroup, whose threads are divided among them, or one of all channels."""
    if images * pixels * C > 12e6:
        images = max(2048, int(12e6 / pixels / C)) + 1
    gen = generator(images + C)
    x = norm.make((images, pixels, C), dtype, gen)
    w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
    kind = norm.ACTIVATIONS[(images + C) % 4]
    y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind)
    norm.check_forward(x, G, w, b, EPS, kind, y, stats)
    g = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
    found = pkg.group_norm_backward(g, x, G, w, b, stats, kind)
    norm.check_backward(g, x, G, w, b, stats, kind, *found)
    inside = torch.full((images + 3, pixels, C), 7.0, device="cuda").to(dtype)          # (what lies behind the last picture stays as it was)
    pkg.group_norm_forward(x, G, w, b, EPS, kind, out=inside[:images])
    assert torch.equal(inside[:images], y) and bool((inside[images:] == 7).all())


def test_a_picture_of_more_than_2_to_the_32_values():
    """Chunks of 2^17 pixels, a thread's 2^12 of them (2^10 steps of its mean): mean off by 2^-12 X, squares by 2^-12; sums of the gradient by 2^-11 of the magnitudes."""
    P, C, G = 2 ** 26 + 77, 64, 2
    gen = generator(2)
    x = torch.empty((1, P, C), dtype=torch.bfloat16, device="cuda")
    for i in range(0, P, 2 ** 22):
        x[:, i:i + 2 ** 22] = torch.randn((1, min(2 ** 22, P - i), C), generator=gen, device="cuda", dtype=torch.bfloat16)
    x[..., 40:] += 0.5
    parts = range(0, P, 2 ** 20)

    def part(t, i):
        return t[0, i:i + 2 ** 20].double().view(-1, G, C // G)
    n = P * C // G
    m = sum(part(x, i).sum((0, 2)) for i in parts) / n
    var = sum((part(x, i) - m[:, None]).square().sum((0, 2)) for i in parts) / n
    r = (var + EPS) ** -0.5
    y, stats = pkg.group_norm_forward(x, G, activation="silu")
    d = 2.0 ** -12 * 8
    assert bool(((stats[0, :, 0].double() - m).abs() <= d).all()) and bool(((stats[0, :, 1].double() / r - 1).abs() <= 2.0 ** -12 + d * d).all())
    for i in parts:
        z = (part(x, i) - stats[0, :, 0].double()[:, None]) * stats[0, :, 1].double()[:, None]
        want = z * torch.sigmoid(z)
        assert bool(((part(y, i) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * (1 + z.abs())).all()), i
    w = torch.linspace(0.5, 1.5, C, device="cuda")
    dx, dw, db = pkg.group_norm_backward(y, x, G, w, torch.zeros(C, device="cuda"), stats, dx=y)      # (g = y, written over)
    x_m, x_r = stats[0, :, 0].double()[:, None], stats[0, :, 1].double()[:, None]
    sums = torch.zeros((4, C), dtype=torch.float64, device="cuda")
    y2, _ = pkg.group_norm_forward(x, G, activation="silu")
    for i in parts:
        u, g = (part(x, i) - x_m) * x_r, part(y2, i)
        sums += torch.stack([(g * u).sum(0), g.sum(0), (g * u).abs().sum(0), g.abs().sum(0)]).view(4, C)
    assert bool(((dw.double() - sums[0]).abs() <= 2.0 ** -11 * sums[2]).all()) and bool(((db.double() - sums[1]).abs() <= 2.0 ** -11 * sums[3]).all())
    of_w = (sums * w.double()).view(4, G, -1).sum(-1) / n
    for i in parts:
        u, g = (part(x, i) - x_m) * x_r, part(y2, i) * w.double().view(G, -1)
        want = x_r * (g - of_w[1][:, None] - u * of_w[0][:, None])
        slack = x_r * (2.0 ** -18 * g.abs() + 2.0 ** -11 * (of_w[3][:, None] + u.abs() * of_w[2][:, None]))
        assert bool(((part(dx, i) - want).abs() <= 2.0 ** -8 * want.abs() + slack).all()), i


@pytest.mark.parametrize("scale", [2.0 ** -50, 2.0 ** -20, 2.0 ** 20, 2.0 ** 40])
def test_small_and_large_numbers(scale):
    """Powers of two: without eps, the result of x * scale is that of x as long as squares stay in range (|x|^2 a group's number of values below 2^127)."""
    for shape, G in (((2, 7, 7, 64), 8), ((2, 150, 140, 24), 3)):
        x = torch.randn(shape, generator=generator(3), device="cuda")
        y, stats = pkg.group_norm_forward(x, G, eps=0.0)
        z, other = pkg.group_norm_forward(x * scale, G, eps=0.0)
        assert torch.equal(other[..., 0], stats[..., 0] * scale) and bool((other[..., 1] * scale / stats[..., 1] - 1).abs().max() <= 2.0 ** -22) and bool((y - z).abs().max() <= 2.0 ** -18)
        found, again = (pkg.group_norm_backward(x, v, G, None, None, s)[0] for v, s in ((x, stats), (x * scale, other)))
        assert bool(((again * scale - found).abs() <= 2.0 ** -13 * (1 + found.abs())).all())


def test_the_largest_numbers_of_half():
    x = (torch.randn((2, 9, 9, 32), generator=generator(4), device="cuda") * 20000).clamp(-65504, 65504).half()
    y, stats = pkg.group_norm_forward(x, 4, activation="relu")
    norm.check_forward(x, 4, None, None, EPS, "relu", y, stats)
    g = x.flip(0)
    norm.check_backward(g, x, 4, None, None, stats, "relu", *pkg.group_norm_backward(g, x, 4, None, None, stats, "relu"))


def test_activations_far_out():
    """z of any size: 0 below, z itself above, NaN stays."""
    x = torch.randn((1, 4, 4, 8), generator=generator(5), device="cuda")
    for kind in ("relu", "silu", "gelu"):
        for z in (-3e38, -1e4, -200.0, -90.0, 90.0, 200.0, 1e4, 3e38):
            y = pkg.group_norm(x, 2, torch.zeros(8, device="cuda"), torch.full((8,), z, device="cuda"), activation=kind)
            assert bool((y == z).all() if z > 0 else (y.abs() <= 1e-30).all()), (kind, z)
            _, stats = pkg.group_norm_forward(x, 2)
            dx, dw, db = pkg.group_norm_backward(torch.ones_like(x), x, 2, torch.zeros(8, device="cuda"), torch.full((8,), z, device="cuda"), stats, kind)
            assert not dx.any() and bool(((db - (16 if z > 0 else 0)).abs() <= 1e-30).all()), (kind, z)
        y = pkg.group_norm(x, 2, None, torch.full((8,), float("nan"), device="cuda"), activation=kind)
        assert bool(y.isnan().all())


def test_the_gradient_of_a_bias_has_the_same_bits_every_time():
    """Values of all sizes, so that another order of additions shows: alone, and beside work on another stream."""
    gen = generator(6)
    side, load = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    for T, H, buckets in ((513, 5, pkg.position_buckets(4, 4, 64)), (700, 12, pkg.position_buckets((9, 9, 9))), (64, 3, pkg.position_buckets(2))):
        m, count = buckets
        p = torch.randint(0, 30, (m.shape[0], 2, T), generator=gen, device="cuda")
        g = torch.randn((2, H, T, T), generator=gen, device="cuda") * torch.exp2(torch.randint(-60, 60, (2, H, T, T), generator=gen, device="cuda").float())
        first = pkg.position_bias_backward(g, p, m, count)
        places.check_gradient(first, g, *places.pairs(p, p, m, count), count)
        for _ in range(6):
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                load.mul_(1.0)
            assert torch.equal(pkg.position_bias_backward(g, p, m, count), first)


def test_rows_behind_the_last_query_and_between_rows_stay_as_they_were():
    gen = generator(7)
    m, count = pkg.position_buckets((4, 4))
    p = torch.randint(0, 9, (2, 37), generator=gen, device="cuda")
    table = torch.randn((count, 3), generator=gen, device="cuda")
    held = torch.full((3, 40, 48), 7.0, device="cuda")
    pkg.position_bias(table, p, m, out=held[:, :37, :37])
    assert bool((held[:, 37:] == 7).all()) and bool((held[:, :, 37:] == 7).all()) and torch.equal(held[:, :37, :37], pkg.position_bias(table, p, m))
    x = torch.randn((3, 20, 40), generator=gen, device="cuda")
    held = torch.full((4, 25, 44), 7.0, device="cuda")
    pkg.group_norm_forward(x, 4, out=held[:3, :20, 1:41])
    inner = torch.zeros(held.shape, dtype=torch.bool, device="cuda")
    inner[:3, :20, 1:41] = True
    assert bool((held[~inner] == 7).all()) and torch.equal(held[:3, :20, 1:41], pkg.group_norm(x, 4))
    held = torch.full((25, 44), 7.0, device="cuda")
    pkg.dropout(x[0], 0.5, drop.seed_of(), out=held[:20, 3:43])
    assert bool((held[20:] == 7).all()) and bool((held[:, :3] == 7).all()) and bool((held[:, 43:] == 7).all())


def test_a_query_whose_segment_no_key_has():
    """Its row is -inf throughout, its gradient counts for nothing; a padded query's row is 0."""
    m, count = pkg.position_buckets(3)
    p = torch.arange(6, device="cuda")[None]
    table = torch.randn((count, 2), device="cuda")
    s, t = torch.tensor([0, 5, -1, 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"), torch.tensor([0, 0, 1, 1, -1, 2], dtype=torch.int32, device="cuda")
    y = pkg.position_bias(table, p, m, p, s, t)
    assert bool((y[:, [1, 4]] == -float("inf")).all()) and not y[:, [2, 5]].any() and bool(y[:, 0, :2].isfinite().all()) and bool((y[:, 3, [0, 1, 4, 5]] == -float("inf")).all())
    g = torch.full((2, 6, 6), float("nan"), device="cuda")
    g[:, 0, :2] = 1.0
    g[:, 3, 2:4] = 1.0
    assert bool(pkg.position_bias_backward(g, p, m, count, p, s, t).sum() == 2 * 4)


@pytest.mark.parametrize("seed", range(24))
def test_norms_drawn_by_chance(seed):
    rng = np.random.default_rng(100 + seed)
    for _ in range(6):
        G = int(2 ** rng.integers(0, 7) if rng.random() < 0.7 else rng.integers(1, 70))
        C = G * int(2 ** rng.integers(0, 6) if rng.random() < 0.6 else rng.integers(1, 40))
        pixels = int(min(2 ** rng.uniform(0, 14), max(1, 3e6 / C)))
        images = int(max(1, min(rng.integers(1, 40), 4e6 // (C * pixels))))
        dtype, kind = norm.TYPES[rng.integers(3)], norm.ACTIVATIONS[rng.integers(4)]
        gen = generator(seed)
        pad = int(rng.integers(0, 9)) if rng.random() < 0.4 else 0
        x = norm.make((images, pixels, C + pad), dtype, gen)[..., pad:]
        w, b = ((torch.randn(C, generator=gen, device="cuda") + 1).to(dtype if rng.random() < 0.5 else torch.float32) for _ in range(2))
        b = b.to(w.dtype)
        print(images, pixels, C, G, dtype, kind, pad, flush=True)
        y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind)
        norm.check_forward(x, G, w, b, EPS, kind, y, stats)
        g = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
        norm.check_backward(g, x, G, w, b, stats, kind, *pkg.group_norm_backward(g, x, G, w, b, stats, kind))


@pytest.mark.parametrize("seed", range(24))
def test_biases_drawn_by_chance(seed):
    rng = np.random.default_rng(200 + seed)
    for _ in range(4):
        axes, H = int(rng.integers(1, 5)), int(rng.integers(1, 30))
        Q, K = (int(2 ** rng.uniform(0, 10)) for _ in range(2))
        B = None if rng.random() < 0.3 else int(rng.integers(1, 5))
        while (B or 1) * Q * K * H > 6e6:
            Q, K = (Q + 1) // 2, (K + 1) // 2
        exact = [int(rng.integers(1, 40 if axes < 3 else 7)) for _ in range(axes)]
        coarse = [int(rng.integers(0, 6)) for _ in range(axes)]
        far = [e + int(rng.integers(1, 300)) for e in exact]
        buckets, count = pkg.position_buckets(exact, coarse, far, bool(rng.random() < 0.3))
        gen = generator(seed)
        q, k, s, t = places.setting(B, Q, K, axes, rng.random() < 0.5, gen, int(2 ** rng.uniform(1, 9)), torch.int64 if rng.random() < 0.3 else torch.int32)
        dtype = places.TYPES[rng.integers(3)]
        table = torch.randn((count, H), generator=gen, device="cuda").to(dtype if rng.random() < 0.5 else torch.float32)
        print(B, Q, K, H, exact, coarse, far, dtype, flush=True)
        y = pkg.position_bias(table, q, buckets, k, s, t, dtype=dtype)
        bucket, apart = places.pairs(q, k, buckets, count, s, t)
        want = places.bias(table, dtype, bucket, apart)
        assert torch.equal(y.cpu(), want[0] if B is None else want)
        g = torch.randn(y.shape, generator=gen, device="cuda").to(dtype)
        places.check_gradient(pkg.position_bias_backward(g, q, buckets, count, k, s, t), g if B is not None else g[None], bucket, apart, count)


@pytest.mark.parametrize("seed", range(8))
def test_dropouts_drawn_by_chance(seed):
    rng = np.random.default_rng(300 + seed)
    for _ in range(8):
        dim, p = int(2 ** rng.uniform(0, 11)), float(rng.random())
        rows = int(max(1, min(2 ** rng.uniform(0, 12), 1e6 // dim)))
        dtype = drop.TYPES[rng.integers(3)]
        kind = torch.float32 if rng.random() < 0.5 else dtype
        pads = [int(rng.integers(0, 9)) for _ in range(3)]
        gen = generator(seed)
        x, r, out = (torch.randn((rows, dim + a), generator=gen, device="cuda").to(t)[:, a:] for a, t in zip(pads, (dtype, kind, kind)))
        seed_at, call = drop.seed_of(int(rng.integers(-2 ** 62, 2 ** 62)), int(rng.integers(-2 ** 62, 2 ** 62))), int(rng.integers(0, 65536))
        print(rows, dim, dtype, kind, pads, p, call, flush=True)
        pkg.dropout(x, p, seed_at, call, r, out=out)
        drop.check(out, x, p, seed_at, call, r)

"""Group norm with an activation and its gradients against the formulas in 64 bits.

Tolerances, with units of 2^-24 and X the largest |x| of a group, before the one rounding to the result's type (half a unit):
  mean: a thread's running mean of at most 2^4 runs here, a team member's sum of at most 2^7 values, a tree of six: below 2^8 roundings of at most X: 2^-16 X;
  squares around it: as many roundings of terms that are not below 0: 2^-16 of the variance, and the square of the mean's error; r: half of that and a unit or two: with
  d = 2^-16 X, r is off by 2^-16 + d^2 r^2 of itself;
  z = (x - m) r w + b: d r |w| + |u w| (2^-16 + d^2 r^2) + 2^-22 (|u w| + |b|), and an activation 1.13 times that (its slope is at most that) and 2^-21 |z| for exponential, error
  function and products.
  Gradients (m and r are inputs): z is off by e = 2^-22 (|u w| + |b|), a slope by e (its own is below 1) and 2^-20 of itself and of 1, except at a rectifier's 0, which side of it is found;
  h w, and its products with u, by 2^-20 of the magnitude |g w| 1.13, with sums of below 2^9 roundings: dx by 2^-14 r of the sum of the magnitudes of its three terms;
  sums over chunks are made in 64 bits, those inside by at most 2^9 roundings: dw and db 2^-14 of the sum of the magnitudes."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTIVATIONS = [None, "relu", "silu", "gelu"]
EPS = 1e-5


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def activated(z, kind):
    if kind == "relu":
        return torch.where(z <= 0, 0.0, z), torch.where(z <= 0, 0.0, 1.0).to(z.dtype)
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if kind == "gelu":
        under = torch.special.ndtr(z)
        return z * under, under + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    return z, torch.ones_like(z)


def grouped(x, G):
    """[images, pixels, groups, channels of a group] in 64 bits on the host."""
    return x.double().cpu().reshape(x.shape[0], -1, G, x.shape[-1] // G)


def parameters(w, b, C, G):
    w = torch.ones(C, dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(C, dtype=torch.float64) if b is None else b.double().cpu()
    return w.view(G, -1), b.view(G, -1)


def close(got, want, slack, dtype):
    got = got.double().cpu().reshape(want.shape)
    tol = HALF_UNIT[dtype] * want.abs() + TINY[dtype] + slack
    off = (got - want).abs()
    assert bool((off <= tol).all()), (float((off - tol).max()), float((off / tol).max()))


def check_forward(x, G, w, b, eps, kind, y, stats):
    assert y.shape == x.shape and y.dtype == x.dtype and stats.shape == (x.shape[0], G, 2) and stats.dtype == torch.float32
    v = grouped(x, G)
    W, B = parameters(w, b, x.shape[-1], G)
    m = v.mean((1, 3), keepdim=True)
    var = (v - m).square().mean((1, 3), keepdim=True)
    r = (var + eps) ** -0.5
    d = 2.0 ** -16 * v.abs().amax((1, 3), keepdim=True)
    off_r = 2.0 ** -16 + d * d * r * r
    close(stats[..., 0], m[:, 0, :, 0], d[:, 0, :, 0], torch.float32)
    close(stats[..., 1], r[:, 0, :, 0], (off_r * r)[:, 0, :, 0], torch.float32)
    u = (v - m) * r
    z = u * W + B
    off = d * r * W.abs() + (u * W).abs() * off_r + 2.0 ** -22 * ((u * W).abs() + B.abs())
    close(y, activated(z, kind)[0], 1.13 * off + 2.0 ** -21 * z.abs(), x.dtype)


def check_backward(g, x, G, w, b, stats, kind, dx, dw, db):
    assert dx.shape == x.shape and dx.dtype == x.dtype
    C = x.shape[-1]
    v, g = grouped(x, G), grouped(g, G)
    W, B = parameters(w, b, C, G)
    m, r = (stats.double().cpu()[:, None, :, None, i] for i in (0, 1))
    u = (v - m) * r
    z = u * W + B
    h = g * activated(z, kind)[1]
    hw, size = h * W, g.abs() * W.abs() * 1.13
    want = r * (hw - hw.mean((1, 3), keepdim=True) - u * (hw * u).mean((1, 3), keepdim=True))
    terms = size + size.mean((1, 3), keepdim=True) + u.abs() * (size * u.abs()).mean((1, 3), keepdim=True)
    steep = 0.0 if kind in (None, "relu") else 2.0 ** -22 * ((u * W).abs() + B.abs())         # a slope's error for that of z
    more = g.abs() * W.abs() * steep
    terms_more = more + more.mean((1, 3), keepdim=True) + u.abs() * (more * u.abs()).mean((1, 3), keepdim=True)
    close(dx, want, r * (2.0 ** -14 * terms + terms_more), x.dtype)
    assert (dw is None) == (w is None) and (db is None) == (b is None)
    if dw is not None:
        assert dw.dtype == torch.float32 and dw.shape == (C,)
        close(dw, (h * u).sum((0, 1)).view(-1), (g.abs() * (2.0 ** -14 * 1.13 + steep) * u.abs()).sum((0, 1)).view(-1), torch.float32)
    if db is not None:
        close(db, h.sum((0, 1)).view(-1), (g.abs() * (2.0 ** -14 * 1.13 + steep)).sum((0, 1)).view(-1), torch.float32)


SHAPES = [  # x, groups
    ((1, 1, 1, 1), 1), ((2, 1, 1, 8), 8), ((3, 5), 1), ((1, 14, 14, 64), 8), ((2, 3, 7, 45), 3), ((2, 37, 11, 90), 6), ((3, 4, 4, 24), 24), ((5, 9, 16), 4), ((1, 130, 100, 6), 2),
    ((2, 17, 521), 521), ((1, 40, 2304), 32), ((1, 3, 4100), 5), ((2, 7, 7, 512), 32), ((2, 50, 40, 60), 4), ((70, 2, 2, 4), 1), ((1, 150, 150, 32), 8), ((4, 31, 29, 12), 12),
    ((1, 1, 16384), 4096), ((2, 56, 56, 64), 32), ((9, 28, 28, 128), 32),
]


def make(shape, dtype, gen, offset=1.0):
    C = shape[-1]
    x = torch.randn(shape, generator=gen, device="cuda") * (0.5 + torch.rand(C, generator=gen, device="cuda")) + offset * torch.randn(C, generator=gen, device="cuda")
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,G", SHAPES)
def test_norm_and_gradient(shape, G, dtype):
    gen = generator(shape[-1] + G)
    x, C = make(shape, dtype, gen), shape[-1]
    for i, kind in enumerate(ACTIVATIONS):
        parameter = torch.float32 if i % 2 else dtype
        w = None if i == 0 else (1 + 0.3 * torch.randn(C, generator=gen, device="cuda")).to(parameter)
        b = None if i in (0, 3) else (0.3 * torch.randn(C, generator=gen, device="cuda")).to(parameter)
        y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind)
        check_forward(x, G, w, b, EPS, kind, y, stats)
        g = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        found = pkg.group_norm_backward(g, x, G, w, b, stats, kind)
        check_backward(g, x, G, w, b, stats, kind, *found)
        again = pkg.group_norm_backward(g, x, G, w, b, stats, kind)
        assert all(p is q is None or torch.equal(p, q) for p, q in zip(found, again))


@pytest.mark.parametrize("pixels", [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 15, 16, 17, 31, 33])
@pytest.mark.parametrize("C,G", [(1032, 1), (800, 1), (1376, 2), (2048, 1), (2056, 1), (688, 1), (522, 1), (258, 1), (771, 3)])
def test_wide_groups_of_few_pixels(C, G, pixels):
    """Runs of a pixel that do not divide a workgroup's threads: some of them have none, the others more pixels than their share."""
    gen = generator(C + pixels)
    for dtype in TYPES[:2]:
        x = make((2, pixels, C), dtype, gen)
        w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
        y, stats = pkg.group_norm_forward(x, G, w, b, EPS, "silu")
        check_forward(x, G, w, b, EPS, "silu", y, stats)
        g = torch.randn(x.shape, generator=gen, device="cuda").to(dtype)
        check_backward(g, x, G, w, b, stats, "silu", *pkg.group_norm_backward(g, x, G, w, b, stats, "silu"))


@pytest.mark.parametrize("kind", ACTIVATIONS)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_pixels(dtype, kind):
    """More than one chunk of a picture, and more workgroups than pictures."""
    gen = generator(7)
    for shape, G in (((2, 200, 180, 64), 16), ((1, 301, 99, 40), 8), ((3, 64, 65, 96), 1)):
        x = make(shape, dtype, gen)
        w, b = (torch.randn(shape[-1], generator=gen, device="cuda") for _ in range(2))
        y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind)
        check_forward(x, G, w, b, EPS, kind, y, stats)
        g = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        check_backward(g, x, G, w, b, stats, kind, *pkg.group_norm_backward(g, x, G, w, b, stats, kind))


@pytest.mark.parametrize("dtype", TYPES)
def test_values_far_from_0_and_rows_unlike_the_others(dtype):
    """A group's spread is small beside its mean, or one pixel far from all others: the squares are taken around the mean."""
    gen = generator(8)
    x = (torch.randn((2, 30, 30, 16), generator=gen, device="cuda") + 900.0).to(dtype)
    x[1, 0, 0] = 0.0                                           # (as a picture's border)
    for G in (2, 16):
        y, stats = pkg.group_norm_forward(x, G, None, None, EPS, None)
        v = grouped(x, G)
        m = v.mean((1, 3))
        var = (v - m[:, None, :, None]).square().mean((1, 3))
        assert bool(((stats[..., 0].double().cpu() - m).abs() <= 2.0 ** -16 * 900).all())
        d = 2.0 ** -16 * 910
        assert bool(((stats[..., 1].double().cpu() * (var + EPS) ** 0.5 - 1).abs() <= 2.0 ** -16 + d * d / (var + EPS)).all())
        check_forward(x, G, None, None, EPS, None, y, stats)
    same = torch.full((1, 9, 9, 8), 3.25, device="cuda", dtype=dtype)          # no spread at all
    y, stats = pkg.group_norm_forward(same, 2, None, None, EPS, None)
    assert not y.any() and bool(((stats[..., 1] - EPS ** -0.5).abs() <= 2.0 ** -22 * EPS ** -0.5).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,G,pad,shift", [(16, 4, 8, 0), (16, 4, 3, 1), (24, 3, 8, 4), (45, 5, 1, 0), (8, 8, 8, 2)])
def test_strides(C, G, pad, shift, dtype):
    """A slice of channels, storage that begins anywhere, pictures with something between them."""
    gen = generator(C + pad)

    def lying(kind):
        flat = torch.randn(shift + 3 * (6 * 7 * (C + pad) + 5), generator=gen, device="cuda").to(kind)
        return flat[shift:].as_strided((3, 6, 7, C), (6 * 7 * (C + pad) + 5, 7 * (C + pad), C + pad, 1))
    x, g, out, dx = (lying(dtype) for _ in range(4))
    w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
    y, stats = pkg.group_norm_forward(x, G, w, b, EPS, "silu", out=out)
    assert y is out
    check_forward(x, G, w, b, EPS, "silu", y, stats)
    got = pkg.group_norm_backward(g, x, G, w, b, stats, "silu", dx=dx)
    assert got[0] is dx
    check_backward(g, x, G, w, b, stats, "silu", *got)
    kept, want = x.clone(), out.clone()
    assert torch.equal(pkg.group_norm_forward(x, G, w, b, EPS, "silu", out=x)[0], want)        # in place
    x.copy_(kept)
    want = dx.clone()
    assert torch.equal(pkg.group_norm_backward(g, x, G, w, b, stats, "silu", dx=x)[0], want)
    x.copy_(kept)
    assert torch.equal(pkg.group_norm_backward(g, x, G, w, b, stats, "silu", dx=g)[0], want)


def test_channels_last_memory():
    gen = generator(9)
    x = torch.randn((2, 24, 10, 12), generator=gen, device="cuda").to(memory_format=torch.channels_last)
    y = pkg.group_norm(x.permute(0, 2, 3, 1), 6).permute(0, 3, 1, 2)
    want = torch.nn.functional.group_norm(x, 6)
    assert y.is_contiguous(memory_format=torch.channels_last) and bool(((y - want).abs() <= 2.0 ** -16 * (1 + want.abs())).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_infinite_values_stay_in_their_group(dtype):
    gen = generator(10)
    x = make((3, 20, 20, 32), dtype, gen)
    clean, stats = pkg.group_norm_forward(x, 4, None, None, EPS, "relu")
    for v in (float("nan"), float("inf"), -float("inf")):
        bad = x.clone()
        bad[1, 3, 4, 17] = v
        y, s = pkg.group_norm_forward(bad, 4, None, None, EPS, "relu")
        at = torch.zeros_like(x, dtype=torch.bool)
        at[1, :, :, 16:24] = True
        assert bool(y[at].isnan().all()) and torch.equal(y[~at], clean[~at]) and not bool(s[1, 2, 0].isfinite()) and bool(s[1, 2, 1].isnan())       # (a mean may be infinite)
        g = torch.ones_like(x)
        dx, dw, db = pkg.group_norm_backward(g, bad, 4, torch.ones(32, device="cuda"), torch.zeros(32, device="cuda"), s, "silu")
        assert bool(dx[at].isnan().all()) and not bool(dx[~at].isnan().any())
        assert bool(dw[16:24].isnan().all()) and not bool(dw[:16].isnan().any()) and not bool(dw[24:].isnan().any())


def test_a_rectifier_at_its_border():
    """z is exactly 0, or so near that 32 bits do not tell on which side: the slope is that of z in 64 bits."""
    gen = generator(11)
    C, G = 64, 8
    x = torch.randn((2, 40, 40, C), generator=gen, device="cuda")
    w = 1 + 0.3 * torch.randn(C, generator=gen, device="cuda")
    _, stats = pkg.group_norm_forward(x, G)
    u = (x - stats[:, None, None, :, 0].repeat_interleave(C // G, -1)) * stats[:, None, None, :, 1].repeat_interleave(C // G, -1)
    b = -(u[0, 3, 5] * w)                                      # (so that this pixel's z are of the size of a rounding)
    g = torch.randn(x.shape, generator=gen, device="cuda")
    check_backward(g, x, G, w, b, stats, "relu", *pkg.group_norm_backward(g, x, G, w, b, stats, "relu"))


def test_no_pictures_or_pixels():
    w = torch.ones(6, device="cuda", requires_grad=True)
    for shape in ((0, 4, 4, 6), (2, 0, 4, 6), (0, 6)):
        x = torch.empty(shape, device="cuda", requires_grad=True)
        y = pkg.group_norm(x, 3, w, None)
        assert y.shape == x.shape
        y.sum().backward()
        assert x.grad.shape == x.shape and not w.grad.any()


@pytest.mark.parametrize("kind", ACTIVATIONS)
@pytest.mark.parametrize("dtype", TYPES)
def test_differentiation(dtype, kind):
    gen = generator(12)
    x = make((2, 9, 8, 24), dtype, gen).requires_grad_()
    w, b = (torch.randn(24, generator=gen, device="cuda").to(dtype).requires_grad_() for _ in range(2))
    y = pkg.group_norm(x, 4, w, b, activation=kind)
    g = torch.randn((2, 24, 9, 8), generator=gen, device="cuda").to(dtype).permute(0, 2, 3, 1)             # (as it comes from behind a permutation)
    y.backward(g)
    with torch.no_grad():
        y2, stats = pkg.group_norm_forward(x, 4, w, b, activation=kind)
        dx, dw, db = pkg.group_norm_backward(g.contiguous(), x, 4, w, b, stats, kind)
    assert torch.equal(y, y2) and torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(dtype)) and torch.equal(b.grad, db.to(dtype))
    with torch.no_grad():
        assert not pkg.group_norm(x, 4, w, b, activation=kind).requires_grad


@pytest.mark.parametrize("kind", [None, "silu", "gelu"])
def test_gradients_by_differences(kind):
    """d/dt of sum c y(x + t v) from y at t = +-2^-7.  With y off by 2^-18 a value its sum is off by 2^-18 sum |c| at most, the quotient by 2^-11 sum |c|; the third
    derivative along v, whose values are below 4 and which moves u by at most 8, is below 2^11 a value: 2^-14 / 6 of it, 2^-5 sum |c| in all."""
    gen = generator(13)
    shape, G = (2, 6, 5, 16), 4
    x, v, c = (torch.randn(shape, generator=gen, device="cuda").clamp(-4, 4) for _ in range(3))
    w, b = 1 + 0.2 * torch.randn(16, generator=gen, device="cuda"), 0.2 * torch.randn(16, generator=gen, device="cuda")
    y, stats = pkg.group_norm_forward(x, G, w, b, EPS, kind)
    dx, dw, db = pkg.group_norm_backward(c, x, G, w, b, stats, kind)
    t = 2.0 ** -7

    def value(x, w, b):
        return float((pkg.group_norm(x, G, w, b, EPS, kind).double() * c.double()).sum())
    bound = 2.0 ** -5 * float(c.double().abs().sum())
    assert abs((value(x + t * v, w, b) - value(x - t * v, w, b)) / (2 * t) - float((dx.double() * v.double()).sum())) <= bound
    vw, vb = (torch.randn(16, generator=gen, device="cuda") for _ in range(2))
    got = (value(x, w + t * vw, b + t * vb) - value(x, w - t * vw, b - t * vb)) / (2 * t)
    assert abs(got - float((dw.double() * vw.double()).sum() + (db.double() * vb.double()).sum())) <= bound


def test_captured_and_replayed():
    gen = generator(14)
    x, g = make((3, 50, 40, 32), torch.bfloat16, gen), torch.randn((3, 50, 40, 32), generator=gen, device="cuda").bfloat16()
    w, b = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    pkg.group_norm_forward(x, 4, w, b, EPS, "silu")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, stats = pkg.group_norm_forward(x, 4, w, b, EPS, "silu")
        found = pkg.group_norm_backward(g, x, 4, w, b, stats, "silu")
    for seed in range(4):
        new = generator(30 + seed)
        x.copy_(make(x.shape, torch.bfloat16, new))
        g.copy_(torch.randn(g.shape, generator=new, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want_y, want_stats = pkg.group_norm_forward(x, 4, w, b, EPS, "silu")
        want = pkg.group_norm_backward(g, x, 4, w, b, want_stats, "silu")
        assert torch.equal(y, want_y) and torch.equal(stats, want_stats) and all(torch.equal(p, q) for p, q in zip(found, want))


def test_refusals():
    x, w = torch.randn((2, 4, 4, 8), device="cuda"), torch.ones(8, device="cuda")
    _, stats = pkg.group_norm_forward(x, 2)
    f, b = pkg.group_norm_forward, pkg.group_norm_backward
    for call in (lambda: f(x.cpu(), 2), lambda: f(x.double(), 2), lambda: f(x[0, 0, 0], 2), lambda: f(x, 3), lambda: f(x, 0), lambda: f(x, -2), lambda: f(x.transpose(2, 3), 2), lambda: f(x.transpose(1, 2), 2),
                 lambda: f(x[:, ::2, 1:], 2), lambda: f(x, 2, w[:4]), lambda: f(x, 2, w.half()), lambda: f(x, 2, w.cpu()), lambda: f(x.half(), 2, w, w.half()), lambda: f(x, 2, eps=-1.0),
                 lambda: f(x, 2, eps=float("nan")), lambda: f(x, 2, activation="tanh"), lambda: f(x, 2, activation=1), lambda: f(x, 2, out=x.half()), lambda: f(x, 2, out=x[:1]), lambda: f(x, 2, out=x[:1].expand(2, 4, 4, 8)),
                 lambda: f(x, 2, out=x.clone().requires_grad_()), lambda: b(x[:1], x, 2, None, None, stats), lambda: b(x.half(), x, 2, None, None, stats), lambda: b(x, x, 2, None, None, stats[:1]),
                 lambda: b(x, x, 2, None, None, stats.double()), lambda: b(x, x, 4, None, None, stats), lambda: b(x, x, 2, None, None, None), lambda: b(None, x, 2, None, None, stats)):
        with pytest.raises(ValueError):
            call()
    for shape, G in (((1, 2, 16392), 8), ((1, 2, 8192), 8192)):
        with pytest.raises(pkg.PcrError):
            f(torch.zeros(shape, device="cuda"), G)

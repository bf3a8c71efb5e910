"""Rotation by positions of several axes, alone and behind a norm of every head, and the gradients, against the formulas in 64 bits.

Tolerances, u the half unit of the output's type (2^-24, 2^-11, 2^-8 of a value), before any rounding to it everything in 32 bits:
  angle: the position times the frequency as 32-bit floats is the definition's; the angle's fraction of a turn is cut at 2^-32 turns and becomes a 32-bit
  float of at most half a turn: below 2^-22 radians; sine and cosine add two units, the two products and the sum 2^-23 of (|x| + |y|): in all 2^-21 (|x| + |y|);
  norm: a sum of at most 512 squares, at most 32 of them after each other in a lane and a tree of ten: 2^-19 of itself, half of that in the root, and
  some units of 2^-24 for root, quotient and products: 2^-18 of the value, rotation included;
  gradient: products of these: 2^-17 of the sum of the magnitudes of its terms; sums over rows add 2^-24 for every row that a lane adds (at most
  128 here) and for the joins: 2^-16 of the sum of the magnitudes."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
EPS = 1e-6


def turned(x, positions, frequency, axis, adjacent, sign=1.0):
    """float64 on the host: x [batch, tokens, heads, dim], positions [axes, batch, tokens]."""
    n = frequency.numel()
    x = x.double().cpu()
    angle = (positions.cpu()[axis.cpu().long()].float() * frequency.cpu()[:, None, None]).double().permute(1, 2, 0)[:, :, None]
    c, s = torch.cos(angle), torch.sin(angle) * sign
    y = x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def pair_sums(x, n, adjacent):
    """|x| + |y| of each element's pair; |x| behind the pairs."""
    m = x.abs().double().cpu().clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
    both = m[..., a] + m[..., b]
    m[..., a] = both
    m[..., b] = both
    return m


def close(got, want, slack):
    got, want = got.double().cpu(), want
    dtype = slack[0]
    tol = HALF_UNIT[dtype] * want.abs() + TINY[dtype] + slack[1]
    off = (got - want).abs()
    assert got.shape == want.shape and bool((off <= tol).all()), float((off - tol).max())


def make(B, T, Hq, Hk, D, dtype, memory, gen, shift=0):
    """Queries and keys [B, T, heads, D] in one of the ways they lie; shift: elements that the storage begins later."""
    def rand(*shape):
        n = 1
        for v in shape:
            n *= v
        flat = torch.randn(n + shift, generator=gen, device="cuda").to(dtype)
        return flat[shift:].view(shape)
    if memory == "fused":
        x = rand(B, T, (Hq + 2 * Hk) * D)
        return x[..., :Hq * D].unflatten(-1, (Hq, D)), x[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D))
    if memory == "heads":
        return rand(B, Hq, T, D).transpose(1, 2), rand(B, Hk, T, D).transpose(1, 2)
    return rand(B, T, Hq, D), rand(B, T, Hk, D)


def setting(pairs, axes, B, T, gen, far=500, kind=torch.int32):
    each = [pairs // axes] * (axes - 1)
    frequency, axis = pkg.axis_frequencies(each + [pairs - sum(each)], 10000.0)
    positions = torch.randint(-far, far, (axes, B, T), generator=gen, device="cuda", dtype=kind)
    return positions, frequency, axis


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


SHAPES = [  # batch, tokens, qheads, kheads, dim, pairs, axes, memory
    (1, 1, 1, 1, 2, 1, 1, "split"), (1, 1, 32, 8, 128, 64, 3, "split"), (3, 5, 4, 2, 72, 36, 2, "fused"), (2, 130, 7, 1, 80, 40, 3, "heads"),
    (1, 333, 3, 3, 96, 32, 3, "fused"), (2, 7, 5, 1, 72, 18, 2, "split"), (1, 17, 2, 1, 7, 3, 1, "split"), (1, 9, 2, 2, 512, 256, 4, "split"),
    (1, 4, 2, 1, 511, 255, 2, "heads"), (2, 40, 6, 2, 64, 0, 1, "split"), (5, 1, 3, 1, 10, 5, 2, "fused"), (1, 700, 1, 1, 256, 128, 3, "heads"),
    (2, 3, 4, 4, 260, 65, 3, "split"), (1, 2100, 4, 1, 32, 16, 2, "split"), (1, 2, 3, 1, 1, 0, 1, "split"),
]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,T,Hq,Hk,D,pairs,axes,memory", SHAPES)
def test_rotation_and_its_inverse(B, T, Hq, Hk, D, pairs, axes, memory, dtype, adjacent):
    gen = generator(D + T)
    q, k = make(B, T, Hq, Hk, D, dtype, memory, gen)
    positions, frequency, axis = setting(pairs, axes, B, T, gen)
    for inverse in (False, True):
        for x, y in zip((q, k), pkg.rotate_axes(q, k, positions, frequency, axis, adjacent=adjacent, inverse=inverse)):
            close(y, turned(x, positions, frequency, axis, adjacent, -1.0 if inverse else 1.0), (dtype, 2.0 ** -21 * pair_sums(x, pairs, adjacent)))


def norm_parts(x, w):
    x = x.double().cpu()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x, r, (torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double().cpu())


@pytest.mark.parametrize("weights", ["type", "float", "none"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,T,Hq,Hk,D,pairs,axes,memory", SHAPES)
def test_norm_with_rotation_and_its_gradient(B, T, Hq, Hk, D, pairs, axes, memory, dtype, adjacent, weights):
    gen = generator(D + T + 1)
    q, k = make(B, T, Hq, Hk, D, dtype, memory, gen)
    gq, gk = make(B, T, Hq, Hk, D, dtype, "split" if memory == "fused" else "fused", gen)
    positions, frequency, axis = setting(pairs, axes, B, T, gen)
    wq, wk = (None if weights == "none" else (1 + 0.3 * torch.randn(D, generator=gen, device="cuda")).to(torch.float32 if weights == "float" else dtype) for _ in range(2))
    for x, w, y in zip((q, k), (wq, wk), pkg.norm_rotate(q, k, wq, wk, positions, frequency, axis, EPS, adjacent)):
        x, r, w = norm_parts(x, w)
        u = x * r * w
        close(y, turned(u, positions, frequency, axis, adjacent), (dtype, 2.0 ** -18 * pair_sums(u, pairs, adjacent)))
    dq, dk, dwq, dwk = pkg.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, frequency, axis, EPS, adjacent)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        assert (dw is None) == (w is None)
        x, r, w = norm_parts(x, w)
        h, size = turned(g, positions, frequency, axis, adjacent, -1.0), pair_sums(g, pairs, adjacent)
        want = r * (h * w - x * r * r * (h * w * x).mean(-1, keepdim=True))
        terms = r * (size * w.abs() + x.abs() * r * r * (size * (w * x).abs()).mean(-1, keepdim=True))
        close(dx, want, (dtype, 2.0 ** -17 * terms))
        if dw is not None:
            close(dw, (h * x * r).sum((0, 1, 2)), (torch.float32, 2.0 ** -16 * (size * (x * r).abs()).sum((0, 1, 2))))


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_far_positions(kind):
    gen = generator(5)
    q, k = make(2, 6, 2, 1, 32, torch.float32, "split", gen)
    frequency, axis = pkg.axis_frequencies([8, 8], 10000.0)
    far = 2 ** 31 - 1 if kind == torch.int32 else 2 ** 40 + 12345
    positions = torch.tensor([[[0, 1, -1, far, -far, 123456789]] * 2, [[far, 7, 65536, -3, 10 ** 9, 10 ** 9 + 1]] * 2], device="cuda", dtype=kind)
    for x, y in zip((q, k), pkg.rotate_axes(q, k, positions, frequency, axis)):
        close(y, turned(x, positions, frequency, axis, False), (torch.float32, 2.0 ** -21 * pair_sums(x, 16, False)))


def test_positions_for_all_sequences_transposed_positions_and_no_keys():
    gen = generator(6)
    q, _ = make(3, 11, 4, 1, 64, torch.bfloat16, "heads", gen)
    positions, frequency, axis = setting(32, 3, 3, 11, gen)
    shared = positions[:, 0]
    y, none = pkg.rotate_axes(q, None, shared, frequency, axis)
    assert none is None
    assert torch.equal(y, pkg.rotate_axes(q, None, shared[:, None].expand(3, 3, 11), frequency, axis)[0])
    turned_memory = positions.permute(1, 2, 0).contiguous().permute(2, 0, 1)
    assert torch.equal(pkg.rotate_axes(q, None, turned_memory, frequency, axis)[0], pkg.rotate_axes(q, None, positions, frequency, axis)[0])
    packed = q[1]                                              # [tokens, heads, dim]
    assert torch.equal(pkg.rotate_axes(packed, None, positions[:, 1], frequency, axis)[0], pkg.rotate_axes(q, None, positions, frequency, axis)[0][1])


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_any_alignment_gives_the_same(shift):
    gen = generator(7)
    B, T, Hq, Hk, D = 2, 37, 5, 2, 96
    positions, frequency, axis = setting(48, 3, B, T, gen)
    w = torch.randn(D, generator=gen, device="cuda").bfloat16()
    q, k = make(B, T, Hq, Hk, D, torch.bfloat16, "split", gen, shift)
    q0, k0 = q.clone(), k.clone()
    # (a lane's share of a row, and so the order of a sum, goes by the alignment: the norm may round another way)
    for a, b in zip(pkg.rotate_axes(q, k, positions, frequency, axis), pkg.rotate_axes(q0, k0, positions, frequency, axis)):
        assert torch.equal(a, b)
    for x, y in zip((q, k), pkg.norm_rotate(q, k, w, w, positions, frequency, axis, EPS)):
        x, r, v = norm_parts(x, w)
        close(y, turned(x * r * v, positions, frequency, axis, False), (torch.bfloat16, 2.0 ** -18 * pair_sums(x * r * v, 48, False)))


def test_in_place_and_broadcast_gradients():
    gen = generator(8)
    positions, frequency, axis = setting(64, 3, 2, 50, gen)
    w = torch.randn(128, generator=gen, device="cuda")
    for memory in ("split", "fused", "heads"):
        q, k = make(2, 50, 8, 2, 128, torch.bfloat16, memory, gen)
        gq, gk = make(2, 50, 8, 2, 128, torch.bfloat16, "split", gen)
        want = pkg.norm_rotate(q, k, w, w, positions, frequency, axis)
        back = pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
        again = pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis, dq=gq, dk=gk)
        assert all(torch.equal(a, b) for a, b in zip(back, again))
        got = pkg.norm_rotate(q, k, w, w, positions, frequency, axis, q_out=q, k_out=k)
        assert all(torch.equal(a, b) for a, b in zip(want, got)) and got[0] is q and got[1] is k
    one = torch.randn((1, 1, 1, 128), generator=gen, device="cuda").bfloat16()
    wide = one.expand(2, 50, 8, 128), one.expand(2, 50, 2, 128)
    a = pkg.norm_rotate_backward(*wide, q, k, w, w, positions, frequency, axis)
    b = pkg.norm_rotate_backward(*(g.contiguous() for g in wide), q, k, w, w, positions, frequency, axis)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_stream_that_is_named():
    gen = generator(15)
    positions, frequency, axis = setting(32, 3, 4, 64, gen)
    q, k = make(4, 64, 8, 2, 64, torch.bfloat16, "split", gen)
    gq, gk = make(4, 64, 8, 2, 64, torch.bfloat16, "split", gen)
    w = torch.randn(64, generator=gen, device="cuda")
    want = pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
    side = torch.cuda.Stream()
    for stream in (side.cuda_stream, 0):
        side.wait_stream(torch.cuda.current_stream())
        got = pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_sequences_that_are_one_and_sequences_that_are_not():
    """Sequences whose tokens follow each other at one stride are taken as one; with another order of memory, shared positions or a gap between
    sequences they are not: the results are the same."""
    gen = generator(16)
    for T in (1, 37):
        positions, frequency, axis = setting(24, 2, 9, T, gen)
        q, k = make(9, T, 3, 1, 48, torch.float16, "split", gen)
        want = pkg.norm_rotate(q, k, None, None, positions, frequency, axis)
        wide = torch.zeros((9, T + 5, 3, 48), dtype=torch.float16, device="cuda")
        wide[:, 2:2 + T] = q
        assert torch.equal(pkg.norm_rotate(wide[:, 2:2 + T], k, None, None, positions, frequency, axis)[0], want[0])
        across = q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(pkg.norm_rotate(across, k, None, None, positions.transpose(1, 2).contiguous().transpose(1, 2), frequency, axis)[0], want[0])
        shared = positions[:, :1].expand(2, 9, T)
        assert torch.equal(pkg.norm_rotate(q, k, None, None, shared[:, 0], frequency, axis)[1], pkg.norm_rotate(q, k, None, None, shared.contiguous(), frequency, axis)[1])


def test_no_tokens_and_no_heads():
    positions, frequency, axis = setting(8, 2, 1, 0, generator(9))
    w = torch.ones(16, device="cuda")
    q = torch.empty((1, 0, 4, 16), device="cuda")
    assert pkg.rotate_axes(q, q, positions, frequency, axis)[0].shape == q.shape
    assert pkg.norm_rotate(q, None, w, None, positions, frequency, axis)[1] is None
    dq, dk, dwq, dwk = pkg.norm_rotate_backward(q, q, q, q, w, w, positions, frequency, axis)
    assert dq.shape == q.shape and not dwq.any() and not dwk.any()
    positions, frequency, axis = setting(8, 2, 1, 3, generator(9))
    q = torch.empty((1, 3, 0, 16), device="cuda")
    dq, dk, dwq, dwk = pkg.norm_rotate_backward(q, None, q, None, w, None, positions, frequency, axis)
    assert not dwq.any() and dwk is None


def test_infinities_and_nan_stay_in_their_row_and_behind_the_pairs_alone():
    gen = generator(10)
    q = torch.randn((1, 6, 2, 24), generator=gen, device="cuda")
    positions, frequency, axis = setting(8, 2, 1, 6, gen)
    clean = pkg.rotate_axes(q, None, positions, frequency, axis)[0]
    bad = q.clone()
    bad[0, 2, 1, 20] = float("inf")
    bad[0, 2, 1, 21] = float("nan")
    got = pkg.rotate_axes(bad, None, positions, frequency, axis)[0]
    assert torch.isinf(got[0, 2, 1, 20]) and torch.isnan(got[0, 2, 1, 21])
    got[0, 2, 1, 20:22] = clean[0, 2, 1, 20:22]
    assert torch.equal(got, clean)
    w = torch.ones(24, device="cuda")
    a, b = pkg.norm_rotate(q, None, w, None, positions, frequency, axis)[0], pkg.norm_rotate(bad, None, w, None, positions, frequency, axis)[0]
    other = torch.ones(6, 2, dtype=torch.bool)
    other[2, 1] = False
    assert torch.equal(a[0][other], b[0][other])


def test_differentiation_and_differences():
    """Through autograd, float32: along a random direction the loss changes as the gradient says.  Differences over 2 h with h = 2^-7 leave h^2 / 6 of the
    third derivative (the function is smooth at the scale of 1: below 2^-14 of the terms' sum here) and 2^-24 of the loss's terms over h."""
    gen = generator(11)
    positions, frequency, axis = setting(16, 3, 2, 9, gen)
    q, k = (torch.randn((2, 9, h, 40), generator=gen, device="cuda", requires_grad=True) for h in (4, 2))
    wq, wk = (torch.randn(40, generator=gen, device="cuda", requires_grad=True) for _ in range(2))
    cq, ck = (torch.randn((2, 9, h, 40), generator=gen, device="cuda") for h in (4, 2))

    def loss(q, k, wq, wk):
        a, b = pkg.norm_rotate(q, k, wq, wk, positions, frequency, axis)
        a, b = pkg.rotate_axes(a, b, positions, frequency, axis, adjacent=True)
        return ((a * cq).double().sum() + (b * ck).double().sum()), ((a * cq).abs().double().sum() + (b * ck).abs().double().sum())
    at = (q, k, wq, wk)
    loss(*at)[0].backward()
    for j, x in enumerate(at):
        d = torch.randn(x.shape, generator=gen, device="cuda")
        along = (x.grad.double() * d.double()).sum()
        h = 2.0 ** -7
        with torch.no_grad():
            up, size = loss(*(y + h * d if i == j else y for i, y in enumerate(at)))
            down, _ = loss(*(y - h * d if i == j else y for i, y in enumerate(at)))
        assert abs((up - down) / (2 * h) - along) <= (2.0 ** -9 if j < 2 else 2.0 ** -13) * size, (j, float(along), float((up - down) / (2 * h)))


def test_streams_and_graphs():
    """On a stream of the caller's; and captured, replayed between other work, against the eager result every time."""
    gen = generator(12)
    positions, frequency, axis = setting(32, 3, 4, 64, gen)
    q, k = make(4, 64, 8, 2, 64, torch.bfloat16, "fused", gen)
    gq, gk = make(4, 64, 8, 2, 64, torch.bfloat16, "split", gen)
    w = torch.randn(64, generator=gen, device="cuda")
    want = pkg.norm_rotate(q, k, w, w, positions, frequency, axis) + pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = pkg.norm_rotate(q, k, w, w, positions, frequency, axis) + pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = pkg.norm_rotate(q, k, w, w, positions, frequency, axis) + pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
    for turn in range(4):
        q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
        graph.replay()
        want = pkg.norm_rotate(q, k, w, w, positions, frequency, axis) + pkg.norm_rotate_backward(gq, gk, q, k, w, w, positions, frequency, axis)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held)), turn


def test_offsets_past_32_bits():
    """A head's elements lie more than 2^31 elements behind the first one's."""
    gen = generator(13)
    T, D = 3, 64
    far = 2 ** 31 + 64
    held = torch.empty(far + T * D, dtype=torch.bfloat16, device="cuda")
    x = held.as_strided((1, T, 2, D), (0, D, far, 1))
    x.copy_(torch.randn((1, T, 2, D), generator=gen, device="cuda"))
    positions, frequency, axis = setting(32, 3, 1, T, gen)
    want = pkg.rotate_axes(x.contiguous(), None, positions, frequency, axis)[0]
    assert torch.equal(pkg.rotate_axes(x, None, positions, frequency, axis)[0], want)
    pkg.rotate_axes(x, None, positions, frequency, axis, q_out=x)
    assert torch.equal(x, want)


def test_refusals():
    gen = generator(14)
    q, k = make(2, 5, 4, 2, 32, torch.float16, "split", gen)
    positions, frequency, axis = setting(16, 3, 2, 5, gen)
    w = torch.ones(32, device="cuda", dtype=torch.float16)

    def call(**more):
        a = dict(q=q, k=k, q_weight=w, k_weight=w, positions=positions, frequency=frequency, axis=axis)
        a.update(more)
        return pkg.norm_rotate(**a)
    call()
    for bad in (dict(q=q.cpu()), dict(q=q.double(), k=k.double()), dict(k=k.float()), dict(k=k[:, :4]), dict(q=q[0, 0], k=k[0, 0]), dict(q=q.transpose(2, 3), k=None, k_weight=None),
                dict(positions=positions[:, :, :4]), dict(positions=positions.float()), dict(positions=positions.repeat(2, 1, 1)), dict(frequency=frequency.double()),
                dict(axis=axis[:8]), dict(axis=axis.long()), dict(frequency=frequency.repeat(2), axis=axis.repeat(2)), dict(q_weight=w[:31]), dict(q_weight=w.float()), dict(q_weight=w.bfloat16(), k_weight=w.bfloat16()),
                dict(eps=-1.0), dict(k=None), dict(q_out=q[:, :4]), dict(k_out=k.float()), dict(q_out=q[:, :, :1].expand(2, 5, 4, 32)), dict(positions=positions.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    wide = torch.zeros((1, 2, 1, 514), device="cuda", dtype=torch.float16)
    with pytest.raises(pkg.PcrError) as e:
        pkg.rotate_axes(wide, None, positions[:, :1, :2], frequency, axis)
    assert e.value.code == pkg.E_RANGE
    with pytest.raises(ValueError):
        pkg.norm_rotate_backward(q, None, q, k, w, w, positions, frequency, axis)
    with pytest.raises(ValueError):
        pkg.norm_rotate_backward(q.float(), k, q, k, w, w, positions, frequency, axis)

"""Dropout from counters, onto a residual, against the generator in unsigned integers and the formula in 64 bits.

Tolerance: 1 / (1 - p) as a 32-bit float, its product with x and the sum with the residual are a rounding each, 3 * 2^-24 of the magnitudes; then one rounding to
the result's type (half a unit).  Which elements are dropped has to be equal."""
import numpy as np
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def philox(counter, key):
    """Four words of Philox4x32-10: counter [4][n] and key [2] as unsigned 64-bit integers below 2^32."""
    low, shift = np.uint64(2 ** 32 - 1), np.uint64(32)
    c, k = [np.asarray(v, np.uint64) for v in counter], [int(v) for v in key]
    for i in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        k0, k1 = np.uint64((k[0] + i * 0x9E3779B9) % 2 ** 32), np.uint64((k[1] + i * 0xBB67AE85) % 2 ** 32)
        c = [(b >> shift) ^ c[1] ^ k0, b & low, (a >> shift) ^ c[3] ^ k1, a & low]
    return c


def kept(n, p, seed, call, first=0):
    """Which of the elements first .. first + n - 1 (first a multiple of 4) are kept."""
    key, step = (int(v) % 2 ** 64 for v in seed.tolist())
    group = np.arange(first // 4, first // 4 + (n + 3) // 4, dtype=np.uint64)
    word = philox([group & np.uint64(2 ** 32 - 1), (group >> np.uint64(32)) + np.uint64(65536 * call), np.full_like(group, step % 2 ** 32), np.full_like(group, step >> 32)],
                  [key % 2 ** 32, key >> 32])
    return torch.from_numpy(np.stack(word, 1).reshape(-1)[:n] >= np.uint64(round(p * 2 ** 32)))


def seed_of(key=0x123456789ABCDEF, step=5):
    return torch.tensor([key, step], dtype=torch.int64, device="cuda")


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def check(y, x, p, seed, call, residual=None):
    mask = kept(x.numel(), p, seed, call).view(x.shape)
    part = torch.where(mask, x.double().cpu() / max(1 - p, 1e-300), 0.0)
    beside = torch.zeros_like(part) if residual is None else residual.double().cpu()
    want = part + beside
    tol = HALF_UNIT[y.dtype] * want.abs() + TINY[y.dtype] + 3 * 2.0 ** -24 * (part.abs() + beside.abs())
    off = (y.double().cpu() - want).abs()
    assert y.shape == x.shape and bool((off <= tol).all()), float((off - tol).max())
    if residual is None:
        assert not bool(y.cpu()[~mask].any())


def test_the_generator_gives_the_published_words():
    """The three known answers that are published with the generator."""
    ones = 2 ** 32 - 1
    for counter, key, want in (((0,) * 4, (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((ones,) * 4, (ones, ones), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(w[0]) for w in philox([[v] for v in counter], key)) == want


@pytest.mark.parametrize("residual", ["none", "same", "float"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1,), (3,), (4,), (5,), (7, 1), (2, 8), (3, 9), (5, 16), (2, 3, 5, 7), (13, 1023), (64, 1024), (2050, 129), (1, 100001)])
def test_forward_and_gradient(shape, dtype, residual):
    gen = generator(len(shape) + shape[-1])
    x = torch.randn(shape, generator=gen, device="cuda").to(dtype)
    kind = torch.float32 if residual == "float" else dtype
    r = None if residual == "none" else torch.randn(shape, generator=gen, device="cuda").to(kind)
    seed = seed_of(step=shape[-1])
    for p, call in ((0.1, 0), (0.5, 65535)):
        check(pkg.dropout(x, p, seed, call=call, residual=r), x, p, seed, call, r)
        g = torch.randn(shape, generator=gen, device="cuda").to(kind)
        dx = pkg.dropout_backward(g, p, seed, call=call, dtype=dtype)
        assert dx.dtype == dtype
        check(dx, g, p, seed, call)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad,shift", [(5, 24, 8, 0), (7, 24, 3, 1), (9, 13, 2, 0), (3, 1, 4, 0), (70, 1000, 24, 8), (1, 11, 3, 2), (33, 7, 1, 3), (4, 3, 2, 0)])
def test_rows_with_a_stride(rows, dim, pad, shift, dtype):
    """The mask goes by the elements' indexes, not by where they lie."""
    gen = generator(dim)
    seed = seed_of()

    def strided(kind):
        flat = torch.randn(shift + rows * (dim + pad), generator=gen, device="cuda").to(kind)
        return flat[shift:].view(rows, dim + pad)[:, :dim]
    x, r, f = strided(dtype), strided(dtype), strided(torch.float32)
    assert torch.equal(pkg.dropout(x, 0.3, seed), pkg.dropout(x.contiguous(), 0.3, seed))
    check(pkg.dropout(x, 0.3, seed, residual=r), x, 0.3, seed, 0, r)
    check(pkg.dropout(x, 0.3, seed, residual=f), x, 0.3, seed, 0, f)
    for out, beside in ((strided(dtype), r), (strided(torch.float32), f)):
        whole = out.as_strided((rows, dim + pad), (dim + pad, 1), out.storage_offset())
        before = whole.clone()
        assert pkg.dropout(x, 0.3, seed, residual=beside, out=out) is out
        check(out, x, 0.3, seed, 0, beside)
        assert torch.equal(whole[:, dim:], before[:, dim:])                    # (what is between the rows is left)
    same = x.clone().as_strided(x.shape, (dim, 1)) if rows == 1 else strided(dtype)
    kept_x, want = same.clone(), pkg.dropout(same, 0.3, seed, residual=r)
    assert torch.equal(pkg.dropout(same, 0.3, seed, residual=r, out=same), want) and not torch.equal(same, kept_x)
    want = pkg.dropout(x, 0.3, seed, residual=f)
    assert torch.equal(pkg.dropout(x, 0.3, seed, residual=f, out=f), want)


def test_probabilities_at_their_ends():
    x = torch.randn((50, 37), device="cuda")
    r = torch.randn((50, 37), device="cuda")
    seed = seed_of()
    assert torch.equal(pkg.dropout(x, 0.0, seed), x) and torch.equal(pkg.dropout(x, 0.0, seed, residual=r), x + r)
    assert not pkg.dropout(x, 1.0, seed).any() and torch.equal(pkg.dropout(x, 1.0, seed, residual=r), r)
    assert not pkg.dropout(x, 1.0 - 2.0 ** -60, seed).any()
    for p in (1e-9, 2.0 ** -32, 1 - 2.0 ** -31):
        check(pkg.dropout(x, p, seed), x, p, seed, 0)


def test_what_is_dropped_counts_for_nothing():
    x = torch.full((4, 333), float("nan"), device="cuda")
    x[1] = float("inf")
    seed = seed_of()
    y, mask = pkg.dropout(x, 0.5, seed), kept(x.numel(), 0.5, seed, 0).view(x.shape).cuda()
    assert not y[~mask].any() and bool(y[0][mask[0]].isnan().all()) and bool((y[1][mask[1]] == float("inf")).all())


@pytest.mark.parametrize("key,step", [(0, 0), (-1, -1), (2 ** 63 - 1, 2 ** 32), (-2 ** 63, 2 ** 63 - 1), (2 ** 31, 1)])
def test_keys_and_steps_of_64_bits(key, step):
    x = torch.randn(1001, device="cuda")
    seed = seed_of(key, step)
    check(pkg.dropout(x, 0.4, seed, call=77), x, 0.4, seed, 77)


def test_rates_and_independence():
    """Of n = 2^20 elements a share p is dropped, 6 standard deviations sqrt(p (1 - p) / n) at most off; another step, call or key drops independently of the first:
    the share dropped by both is p^2, within 6 of its own."""
    n = 2 ** 20
    x = torch.ones(n, device="cuda")
    for p in (0.05, 0.3):
        masks = [pkg.dropout(x, p, s, call=c) == 0 for s, c in ((seed_of(), 0), (seed_of(step=6), 0), (seed_of(), 1), (seed_of(key=1), 0))]
        for m in masks:
            assert abs(float(m.double().mean()) - p) < 6 * (p * (1 - p) / n) ** 0.5
        for m in masks[1:]:
            assert abs(float((m & masks[0]).double().mean()) - p * p) < 6 * (p * p * (1 - p * p) / n) ** 0.5


def test_nothing_to_drop():
    seed = seed_of()
    for shape in ((0,), (0, 5), (5, 0), (2, 0, 3)):
        x = torch.empty(shape, device="cuda", requires_grad=True)
        y = pkg.dropout(x, 0.1, seed)
        assert y.shape == x.shape
        y.sum().backward()
        assert x.grad.shape == x.shape


def test_more_than_2_to_the_32_elements():
    """Rows behind the first 2^32 elements: the counters' words and the offsets are of 64 bits."""
    rows, dim = 2 ** 16 + 3, 2 ** 16 + 8
    x = torch.ones((rows, dim), device="cuda", dtype=torch.bfloat16)
    seed = seed_of()
    y = pkg.dropout(x, 0.25, seed, call=3, out=x)
    for row in (0, rows // 2, rows - 3, rows - 1):
        mask = kept(dim, 0.25, seed, 3, row * dim).cuda()
        assert torch.equal(y[row] != 0, mask)
    wide = torch.ones((rows, dim), device="cuda", dtype=torch.bfloat16)[:, :dim - 5]
    y = pkg.dropout(wide, 0.25, seed, call=3, out=wide)
    for row in (0, rows - 4, rows - 1):
        first = row * (dim - 5)
        mask = kept(dim + 4, 0.25, seed, 3, first // 4 * 4)[first % 4:][:dim - 5].cuda()
        assert torch.equal(y[row] != 0, mask)


@pytest.mark.parametrize("residual", ["none", "same", "float"])
@pytest.mark.parametrize("dtype", TYPES)
def test_differentiation(dtype, residual):
    gen = generator(3)
    x = torch.randn((30, 70), generator=gen, device="cuda").to(dtype).requires_grad_()
    kind = torch.float32 if residual == "float" else dtype
    r = None if residual == "none" else torch.randn((30, 70), generator=gen, device="cuda").to(kind).requires_grad_()
    seed = seed_of()
    y = pkg.dropout(x, 0.2, seed, call=9, residual=r)
    g = torch.randn((70, 30), generator=gen, device="cuda").to(kind).T          # (as a transposed view)
    seed[1] += 1                                                                # the gradient goes by the seed that was read
    y.backward(g)
    check(x.grad, g, 0.2, seed_of(), 9)
    assert x.grad.dtype == dtype and (r is None or torch.equal(r.grad, g))
    with torch.no_grad():
        assert not pkg.dropout(x, 0.2, seed).requires_grad


def test_captured_and_replayed():
    """A graph that counts its step up drops other elements at every replay, in the gradient, too."""
    x = torch.randn((40, 100), device="cuda")
    g, seed = torch.randn_like(x), seed_of(step=0)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    pkg.dropout(x, 0.5, seed, out=y)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pkg.dropout(x, 0.5, seed, out=y)
        dx.copy_(pkg.dropout_backward(g, 0.5, seed))
        seed[1] += 1
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        now = seed_of(step=step)
        check(y, x, 0.5, now, 0)
        check(dx, g, 0.5, now, 0)
        torch.randn(1000, device="cuda").sum().item()


def test_refusals():
    x, seed = torch.randn((4, 6), device="cuda"), seed_of()
    r = torch.randn((4, 6), device="cuda")
    for call in (lambda: pkg.dropout(x.double(), 0.1, seed), lambda: pkg.dropout(x.cpu(), 0.1, seed), lambda: pkg.dropout(x, 0.1, seed.cpu()), lambda: pkg.dropout(x, 0.1, seed.int()),
                 lambda: pkg.dropout(x, 0.1, seed[:1]), lambda: pkg.dropout(x, -0.1, seed), lambda: pkg.dropout(x, 1.1, seed), lambda: pkg.dropout(x, float("nan"), seed),
                 lambda: pkg.dropout(x, 0.1, seed, call=-1), lambda: pkg.dropout(x, 0.1, seed, call=65536), lambda: pkg.dropout(x, 0.1, seed, residual=r[:2]),
                 lambda: pkg.dropout(x, 0.1, seed, residual=r.half()), lambda: pkg.dropout(x.T, 0.1, seed), lambda: pkg.dropout(x, 0.1, seed, residual=r.T.contiguous().T),
                 lambda: pkg.dropout(x.half(), 0.1, seed, residual=r.bfloat16()), lambda: pkg.dropout(x, 0.1, seed, out=torch.empty((6, 4), device="cuda")),
                 lambda: pkg.dropout(x, 0.1, seed, residual=r, out=x.half()), lambda: pkg.dropout(x, 0.1, seed, out=x[:1].expand(4, 6)), lambda: pkg.dropout(x, 0.1, None),
                 lambda: pkg.dropout(torch.tensor(1.0, device="cuda"), 0.1, seed), lambda: pkg.dropout_backward(x, 0.1, seed, dtype=torch.float64),
                 lambda: pkg.dropout_backward(x.half(), 0.1, seed, dtype=torch.bfloat16), lambda: pkg.dropout(x, 0.1, seed, out=x.clone().requires_grad_())):
        with pytest.raises(ValueError):
            call()

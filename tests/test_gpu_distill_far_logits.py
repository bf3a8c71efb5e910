"""Gradients of rows whose logits are all far from 0 (all at a mask's value, or around an offset), where 32 bits hold little or nothing of a sum's logarithm
beside the maximum: from saved sums, in one pass with the loss, and through automatic differentiation, on every route that rows of a size take.

Tolerance: as for other rows, half a unit of the output's type and 2^-16 of the magnitude of the gradient's terms (2^-17 of the sums; 2^-17 for the argument of
the exponential: the difference to the maximum is rounded once, to 2^-24 of itself, and times 1 / T once more, with 16 at most where the exponential counts;
saved sums below 128 are off by two roundings of 2^-18)."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -125, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -125}
A_PART, B_PART = 0.7, 0.3


def gradient(z, index, t, labels, T, weight):
    """(gradient, magnitude of its terms) in 64 bits: probabilities from differences to the row's maximum."""
    z = z.double()
    V = z.shape[1]
    d = z - z.max(1, keepdim=True).values
    counts = index >= 0
    p = torch.softmax(torch.where(counts, t.double() / T, -1e300), 1) * counts
    teacher = torch.zeros_like(z).scatter_add_(1, index.clamp(min=0).long(), p)
    q = torch.softmax(d / T, 1) * p.sum(1, keepdim=True)
    there = ((labels >= 0) & (labels < V)).double()[:, None]
    named = torch.zeros_like(z).scatter_(1, labels.clamp(min=0)[:, None], 1.0)
    q1 = torch.softmax(d, 1)
    w = weight.double()[:, None]
    grad = w * (A_PART * T * (q - teacher) + B_PART * there * (q1 - named))
    size = w.abs() * (A_PART * T * (q + teacher) + B_PART * there * (q1 + named))
    return grad, size


def near(got, grad, size):
    tol = HALF_UNIT[got.dtype] * grad.abs() + TINY[got.dtype] + 2.0 ** -16 * size
    off = (got.double() - grad).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), (bad.any(1).nonzero().flatten()[:8].tolist(), float((off - tol).nan_to_num(nan=1e300).max()))


def make(N, V, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + V)
    z = torch.randn((N, V), generator=gen, device="cuda") * 2
    low = torch.finfo(dtype).min
    masked = torch.arange(V, device="cuda") % 3 == 1
    for n in range(N):                                         # by turns: as usual, all at a mask's value, around offsets, far and masked in part
        kind = n % 8
        if kind == 1:
            z[n] = low
        elif kind == 2:
            z[n] = -60000.0 if dtype == torch.float16 else -1e9
        elif kind in (3, 4, 5):
            z[n] += (120.0, 30000.0, -250.0)[kind - 3]
        elif kind == 6:
            z[n] = torch.where(masked, low, z[n] + 5000)
    z = z.to(dtype)
    index = torch.randint(0, V, (N, 12), generator=gen, device="cuda", dtype=torch.int32)
    index[:, 3] = index[:, 8]                                  # twice
    index[:, 5] = -1
    t = (torch.randn((N, 12), generator=gen, device="cuda") * 3).to(dtype)
    labels = torch.randint(0, V, (N,), generator=gen, device="cuda")
    labels[::5] = -100
    labels[1::7] = index[1::7, 0].long()
    weight = torch.rand(N, generator=gen, device="cuda") + 0.25
    return z, index, t, labels, weight


@pytest.mark.parametrize("T", [1.0, 1.5, 2.0, 4.0, 7.0])
@pytest.mark.parametrize("N,V,dtype", [(1600, 300, torch.float32), (1600, 300, torch.bfloat16), (1100, 4000, torch.float16), (17, 2000, torch.float32), (9, 30011, torch.bfloat16),
                                       (40, 9000, torch.float16), (11, 200001, torch.bfloat16), (16, 90001, torch.float32), (400, 100003, torch.float32), (514, 156001, torch.float16),
                                       (140, 140000, torch.bfloat16), (520, 20011, torch.bfloat16)])
def test_gradients_of_rows_far_from_zero(N, V, dtype, T):
    z, index, t, labels, weight = make(N, V, dtype)
    how = dict(labels=labels, temperature=T, distill_part=A_PART, label_part=B_PART)
    grad, size = gradient(z, index, t, labels, T, weight)
    loss, step = pkg.distill_step(z, index, t, weight, **how)
    near(step, grad, size)
    first, sums = pkg.distill_forward(z, index, t, **how)
    back = pkg.distill_backward(weight, z, index, t, sums, **how)
    near(back, grad, size)
    x = z.clone().requires_grad_()
    pkg.distill_loss(x, index, t, **how).backward(weight)
    assert torch.equal(x.grad, back)
    over = z.clone()
    pkg.distill_backward(weight, over, index, t, sums, out=over, **how)
    assert torch.equal(over, back)
    over = z.clone()
    pkg.distill_step(over, index, t, weight, out=over, **how)
    assert torch.equal(over, step)

"""Differentiation of calls on a stream that is named: the same gradients as on the current stream."""
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_the_same_gradients_on_a_named_stream(norm, keys, own):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    frequency, axis = pkg.axis_frequencies((0, 16, 16))
    positions = torch.randint(0, 50, (3, 2, 40), generator=gen, device="cuda")
    q, k = (torch.randn((2, 40, h, 64), generator=gen, device="cuda").bfloat16() for h in (6, 2))
    w = [torch.randn(64, generator=gen, device="cuda") for _ in range(2)]
    cq, ck = (torch.randn(x.shape, generator=gen, device="cuda").bfloat16() for x in (q, k))
    side = torch.cuda.Stream()

    def gradients(stream):
        leaves = [x.clone().requires_grad_() for x in (q, k, *w)]
        a, b, wq, wk = leaves
        torch.cuda.synchronize()
        if norm:
            y, z = pkg.norm_rotate(a, b if keys else None, wq, wk if keys else None, positions, frequency, axis, stream=stream)
        else:
            y, z = pkg.rotate_axes(a, b if keys else None, positions, frequency, axis, stream=stream)
        torch.cuda.synchronize()
        assert y.requires_grad and (z is None or z.requires_grad)
        loss = (y * cq).sum() if z is None else (y * cq).sum() + (z * ck).sum()
        loss.backward()
        torch.cuda.synchronize()
        return [y, z] + [x.grad for x in leaves]
    for got, want in zip(gradients(side.cuda_stream if own else 0), gradients(None)):
        assert (got is None) == (want is None) and (got is None or torch.equal(got, want))
    with torch.no_grad():
        assert not pkg.rotate_axes(q.clone().requires_grad_(), None, positions, frequency, axis, stream=side.cuda_stream)[0].requires_grad

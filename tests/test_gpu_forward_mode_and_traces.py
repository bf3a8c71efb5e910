"""Derivatives of forward mode and traces, which the operators do not have, are refused and not lost."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu


def test_derivatives_of_forward_mode_are_refused():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    frequency, axis = pkg.axis_frequencies((8, 8))
    positions = torch.randint(0, 50, (2, 5), generator=gen, device="cuda")
    q, k = (torch.randn((5, h, 32), generator=gen, device="cuda") for h in (4, 2))
    w = torch.ones(32, device="cuda")
    z, t = torch.randn((6, 40), generator=gen, device="cuda"), torch.randn((6, 3), generator=gen, device="cuda")
    index, weight = torch.randint(0, 40, (6, 3), generator=gen, device="cuda"), torch.ones(6, device="cuda")
    with forward_ad.dual_level():
        def dual(x):
            return forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: pkg.rotate_axes(dual(q), k, positions, frequency, axis), lambda: pkg.rotate_axes(q, dual(k), positions, frequency, axis),
                     lambda: pkg.rotate_axes(q, k, positions, dual(frequency), axis), lambda: pkg.norm_rotate(q, k, dual(w), w, positions, frequency, axis),
                     lambda: pkg.norm_rotate_backward(dual(q), k, q, k, w, w, positions, frequency, axis), lambda: pkg.distill_forward(dual(z), index, t),
                     lambda: pkg.distill_step(z, index, dual(t), weight), lambda: pkg.distill_step(dual(z), index, t, weight)):
            with pytest.raises(ValueError):
                call()
        with pytest.raises(Exception):
            pkg.distill_loss(dual(z), index, t)
        assert torch.equal(pkg.rotate_axes(q, k, positions, frequency, axis)[0], pkg.rotate_axes(q, None, positions, frequency, axis)[0])


def test_traces_are_refused():
    frequency, axis = pkg.axis_frequencies((8, 8))
    positions = torch.arange(10, device="cuda").view(2, 5)
    q = torch.randn((5, 4, 32), device="cuda")
    z, t, index = torch.randn((6, 40), device="cuda"), torch.randn((6, 3), device="cuda"), torch.zeros((6, 3), dtype=torch.int32, device="cuda")
    for f, x in ((lambda x: pkg.rotate_axes(x, None, positions, frequency, axis)[0], q), (lambda x: pkg.norm_rotate(x, None, None, None, positions, frequency, axis)[0], q),
                 (lambda x: pkg.distill_loss(x, index, t), z), (lambda x: pkg.distill_forward(x, index, t)[0], z)):
        with pytest.raises(RuntimeError):
            torch.jit.trace(f, (x,), check_trace=False)
        f(x)

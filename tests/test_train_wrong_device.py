"""Tensors that are not on a GPU, and what is no tensor, are a wrong argument also where a stream is named."""
import pytest
import torch

import paper_1911_00472_amd as pkg

Q, W = torch.zeros((5, 4, 32)), torch.ones(32)
AT = (torch.zeros((1, 5), dtype=torch.int32), torch.ones(8), torch.zeros(8, dtype=torch.int32))
Z, INDEX, TOP, ROW, SUMS = torch.zeros((6, 40)), torch.zeros((6, 3), dtype=torch.int32), torch.zeros((6, 3)), torch.ones(6), torch.zeros((6, 2))
PIXELS, SHAPES, OFFSETS = torch.zeros(12, dtype=torch.uint8), torch.tensor([[2, 2]], dtype=torch.int32), torch.tensor([0, 12])
CALLS = {
    "rotate_axes": lambda s: pkg.rotate_axes(Q, Q, *AT, stream=s),
    "rotate_axes of a leaf": lambda s: pkg.rotate_axes(Q.clone().requires_grad_(), None, *AT, stream=s),
    "rotate_axes of nothing": lambda s: pkg.rotate_axes(None, None, *AT, stream=s),
    "rotate_axes of a list": lambda s: pkg.rotate_axes([1.0], None, None, None, None, stream=s),
    "norm_rotate": lambda s: pkg.norm_rotate(Q, None, W, None, *AT, stream=s),
    "norm_rotate_backward": lambda s: pkg.norm_rotate_backward(Q, Q, Q, Q, W, W, *AT, stream=s),
    "distill_forward": lambda s: pkg.distill_forward(Z, INDEX, TOP, stream=s),
    "distill_backward": lambda s: pkg.distill_backward(ROW, Z, INDEX, TOP, SUMS, stream=s),
    "distill_step": lambda s: pkg.distill_step(Z, INDEX, TOP, ROW, stream=s),
    "patch_rows": lambda s: pkg.patch_rows(PIXELS, SHAPES, OFFSETS, OFFSETS, 1, 2, (0.0,) * 3, (1.0,) * 3, stream=s),
}


@pytest.mark.parametrize("stream", [None, 0, 64])
@pytest.mark.parametrize("name", CALLS)
def test_refused_as_a_wrong_argument(name, stream):
    with pytest.raises(ValueError):
        CALLS[name](stream)

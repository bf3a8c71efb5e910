"""Layers whose tensors are all on the host, on a named stream, too: a wrong argument, told before anything is enqueued."""
import pytest
import torch

import paper_1911_00472_amd as pkg

X, W, STATS, SEED = torch.zeros(2, 3, 8), torch.ones(8), torch.zeros(2, 2, 2), torch.zeros(2, dtype=torch.int64)
TABLE, POSITIONS, BUCKETS, GRAD = torch.zeros(9, 2), torch.zeros((2, 5), dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, 5, 5)
CALLS = {
    "group_norm_forward": lambda s: pkg.group_norm_forward(X, 2, stream=s),
    "group_norm": lambda s: pkg.group_norm(X, 2, W.clone().requires_grad_(), stream=s),
    "group_norm of a list": lambda s: pkg.group_norm([1.0], 2, stream=s),
    "group_norm_backward": lambda s: pkg.group_norm_backward(X, X, 2, W, None, STATS, stream=s),
    "position_bias": lambda s: pkg.position_bias(TABLE, POSITIONS, BUCKETS, stream=s),
    "position_bias with a gradient": lambda s: pkg.position_bias(TABLE.clone().requires_grad_(), POSITIONS, BUCKETS, stream=s),
    "position_bias_backward": lambda s: pkg.position_bias_backward(GRAD, POSITIONS, BUCKETS, 9, stream=s),
    "dropout": lambda s: pkg.dropout(X, 0.5, SEED, stream=s),
    "dropout with a gradient": lambda s: pkg.dropout(X.clone().requires_grad_(), 0.5, SEED, stream=s),
    "dropout_backward": lambda s: pkg.dropout_backward(X, 0.5, SEED, stream=s),
}


@pytest.mark.parametrize("stream", [None, 0, 64])
@pytest.mark.parametrize("name", CALLS)
def test_refused_as_a_wrong_argument(name, stream):
    with pytest.raises(ValueError):
        CALLS[name](stream)

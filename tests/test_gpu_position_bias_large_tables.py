"""The gradient of a table of which its shares' sums would not fit 4 GiB: fewer shares, the same sums."""
import pytest
import torch

import paper_1911_00472_amd as pkg
import test_gpu_position_bias as places

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count,H,T", [(2 ** 21 + 7, 24, 1500), (2 ** 24, 2, 300)])
def test_a_large_table(count, H, T):
    gen = places.generator(count % 1000)
    reach = 40000
    buckets = torch.randint(0, count, (1, 2 * reach + 1), generator=gen, device="cuda", dtype=torch.int32)
    p = torch.randint(-reach // 2, reach // 2, (1, T), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.randn((H, T, T), generator=gen, device="cuda").bfloat16()
    got = pkg.position_bias_backward(g, p, buckets, count)
    bucket = buckets[0].long()[(p[0, None, :].long() - p[0, :, None]).clamp(-reach, reach) + reach].view(-1)
    want = torch.zeros((count, H), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    want.index_add_(0, bucket, g.view(H, -1).T.double())
    size.index_add_(0, bucket, g.view(H, -1).T.double().abs())
    # each share's sum, and the last, rounded to 32 bits
    assert bool(((got.double() - want).abs() <= 2.0 ** -23 * size).all())
    assert torch.equal(got, pkg.position_bias_backward(g, p, buckets, count))

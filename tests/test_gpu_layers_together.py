"""A record decoded, cut into patch rows, and a step of a network on them: group norm with an activation over each picture's map, attention with a bias for the patches' relative places in
pictures packed behind each other, dropout onto the residual; everything between is torch's.  Result and gradients against the same network in 64 bits on the host.

Tolerance: float32 throughout; every product of matrices and every operator is off by at most 2^-14 of the sum of its terms' magnitudes, there are below 2^4 of them
after each other, and what they make of an error is below 2^3 times as large: 2^-7 of the largest value of each result."""
import pytest
import torch

import paper_1911_00472_amd as pkg
from test_gpu_dropout import kept
from test_gpu_position_bias import bias as bias_in_64
from test_gpu_position_bias import pairs

pytestmark = pytest.mark.gpu
PATCH, WIDTH, HEADS, GROUPS, P = 14, 48, 4, 8, 0.25


def parameters():
    gen = torch.Generator()
    gen.manual_seed(3)
    buckets, count = pkg.position_buckets((1, 6, 6), (0, 2, 2), (0, 20, 20))
    shapes = {"into": (WIDTH, 3 * PATCH * PATCH), "weight": (WIDTH,), "bias": (WIDTH,), "qkv": (3 * WIDTH, WIDTH), "table": (count, HEADS), "out": (WIDTH, WIDTH)}
    values = {k: torch.randn(s, generator=gen, dtype=torch.float64) * (s[-1] ** -0.5 if len(s) == 2 and k != "table" else 0.3) for k, s in shapes.items()}
    values["weight"] += 1
    return values, buckets, count


def network(rows, first, values, norm, biased, drop):
    x = rows @ values["into"].T
    y = torch.cat([norm(x[None, a:b], values["weight"], values["bias"])[0] for a, b in zip(first[:-1], first[1:]) if b > a])
    q, k, v = (y @ values["qkv"].T).view(-1, 3, HEADS, WIDTH // HEADS).permute(1, 2, 0, 3).contiguous()
    scores = torch.stack([q[h] @ k[h].T.contiguous() for h in range(HEADS)]) * (WIDTH // HEADS) ** -0.5 + biased(values["table"])
    weight = scores.softmax(-1)
    mixed = torch.stack([weight[h] @ v[h] for h in range(HEADS)]).transpose(0, 1).reshape(-1, WIDTH)
    return drop(mixed @ values["out"].T, y)


def near(got, want, what):
    off, size = float((got.double().cpu() - want).abs().max()), float(want.abs().max())
    assert got.shape == want.shape and off <= 2.0 ** -7 * size, (what, off, size)


@pytest.mark.parametrize("scans", [1, 10])
def test_a_step_on_a_record(rgb_small, scans):
    values, buckets, count = parameters()
    with pkg.pcr_open(rgb_small[0], 0) as record:
        layout = record.patch_layout(PATCH)
        first = layout[2].tolist()
        rows, positions = pkg.patch_rows(record.decode_batch(scans), *layout, PATCH, (0.45,) * 3, (4.0,) * 3, dtype=torch.float32)
    many = min(len(first) - 1, next((i for i, n in enumerate(first) if n > 900), len(first)))      # (as many pictures as 64 bits on the host take)
    first = first[:many + 1]
    n = first[-1]
    rows, positions = rows[:n].contiguous(), positions[:, :n]
    segments = torch.repeat_interleave(torch.arange(many, dtype=torch.int32, device="cuda"), torch.tensor([b - a for a, b in zip(first, first[1:])], device="cuda"))
    seed = torch.tensor([11, 4], device="cuda")
    target = torch.randn((n, WIDTH), generator=torch.Generator().manual_seed(9), dtype=torch.float64)

    ours = {k: v.float().cuda().requires_grad_() for k, v in values.items()}
    got = network(rows, first, ours, lambda x, w, b: pkg.group_norm(x, GROUPS, w, b, activation="silu"), lambda t: pkg.position_bias(t, positions, buckets, segments=segments),
                  lambda x, r: pkg.dropout(x, P, seed, call=1, residual=r))
    loss = (got - target.float().cuda()).square().sum()
    loss.backward()

    plain = {k: v.float().double().requires_grad_() for k, v in values.items()}
    bucket, apart = pairs(positions, positions, buckets, count, segments, segments)
    mask = kept(n * WIDTH, P, seed, 1).view(n, WIDTH)

    def norm(x, w, b):
        return torch.nn.functional.silu(torch.nn.functional.group_norm(x.transpose(1, 2), GROUPS, w, b, 1e-5).transpose(1, 2))

    def biased(table):
        whole = torch.cat([table, torch.zeros((1, HEADS), dtype=torch.float64)])[bucket[0]].permute(2, 0, 1)
        assert torch.equal(bias_in_64(table.detach(), torch.float64, bucket, apart)[0].isinf(), apart.expand(HEADS, -1, -1))
        return whole.masked_fill(apart, -float("inf"))
    want = network(rows.double().cpu(), first, plain, norm, biased, lambda x, r: r + torch.where(mask, x / (1 - P), 0.0))
    (want - target).square().sum().backward()
    near(got.detach(), want.detach(), "result")
    for k in values:
        near(ours[k].grad, plain[k].grad, k)

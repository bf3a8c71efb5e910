"""Layers of a network that trains on decoded pictures, between its matrix products: what is timed, in a plain form and through the package.

Feature maps behind the first convolutions are normalised by groups of channels and go through an activation, channels last as pictures are
decoded; attention over patch rows adds a learned bias for the relative position of its tokens (row, column, frame), counted in buckets; what a branch gives
goes through dropout onto the residual stream.  A case is a dict of plain values:

  op        norm      group norm and activation, with the statistics that its gradient takes; `backward`: the gradients of input, weight and bias
            bias      bias [batch, heads, queries, keys] from a table [buckets, heads]; `backward`: the table's gradient
            dropout   what is kept of x over its probability, added to a residual; `backward`: the gradient of x
  dtype     of what is read and written
  norm:     images, height, width, channels, groups, activation (none, relu, silu, gelu)
  bias:     batch, queries, keys, heads, axes; exact, coarse, far (distances below `exact` have a bucket each, those up to `far` share `coarse` buckets that
            widen by a constant factor, on either side of every axis), one_sided (keys ahead count as distance 0), packed (several pictures in
            a sequence, which do not see each other, and padding behind them)
  dropout:  rows, dim, p, residual (none; same: of x's type; float: of 32 bits, as the result then)

The random numbers of dropout are those of the counter-based generator Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011):
element e takes word e mod 4 of the generator's output for the key `seed` and the counter (e / 4, call, step); it is dropped where that is below p 2^32.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-5
SMALLEST = 1.0e4
LARGEST = {"norm": 3.0e8, "bias": 4.0e8, "dropout": 3.3e8}    # bytes that a drawn case moves at most


def _norm(name, images, size, channels, groups, activation, dtype, backward=False):
    return {"name": name, "op": "norm", "images": images, "height": size[0], "width": size[1], "channels": channels, "groups": groups, "activation": activation,
            "backward": backward, "dtype": dtype}


def _bias(name, batch, queries, keys, heads, axes, buckets, dtype, one_sided=False, packed=False, backward=False):
    return {"name": name, "op": "bias", "batch": batch, "queries": queries, "keys": keys, "heads": heads, "axes": axes, "exact": buckets[0], "coarse": buckets[1],
            "far": buckets[2], "one_sided": one_sided, "packed": packed, "backward": backward, "dtype": dtype}


def _dropout(name, rows, dim, p, residual, dtype, backward=False):
    return {"name": name, "op": "dropout", "rows": rows, "dim": dim, "p": p, "residual": residual, "backward": backward, "dtype": dtype}


def listed():
    return [
        # one picture that is being answered: launches and latency
        _norm("norm_one", 1, (14, 14), 64, 8, "relu", "float16"),
        # crops of 224 behind a first convolution of stride 2, few channels to a group
        _norm("norm_stem", 64, (112, 112), 64, 32, "silu", "bfloat16"),
        # a few pictures of an odd size in 32 bits, channels that are not whole 16-byte runs
        _norm("norm_odd", 5, (37, 53), 90, 6, "gelu", "float32"),
        # gradient in the middle of a network
        _norm("norm_backward", 64, (56, 56), 256, 32, "silu", "bfloat16", backward=True),
        # a new token of 32 sequences that are being answered, against all before it
        _bias("bias_token", 32, 1, 4099, 16, 1, (16, 16, 128), "bfloat16", one_sided=True),
        # sequences into which pictures of many sizes are packed, a bucket for each difference of rows and columns
        _bias("bias_packed", 16, 1024, 1024, 12, 2, (32, 0, 0), "float16", packed=True),
        # gradient of one window of 8 x 8 patches: few elements, many buckets
        _bias("bias_window_backward", 1, 64, 64, 6, 2, (8, 0, 0), "float32", backward=True),
        # gradient over a long sequence of lines: many elements in few buckets
        _bias("bias_long_backward", 1, 4096, 4096, 12, 1, (8, 8, 128), "bfloat16", backward=True),
        # gradient over packed pictures: a bucket for each difference
        _bias("bias_packed_backward", 4, 1501, 1501, 12, 2, (32, 0, 0), "bfloat16", packed=True, backward=True),
        # a token each of 32 sequences
        _dropout("dropout_few", 32, 1024, 0.1, "same", "bfloat16"),
        # a branch in 16 bits onto a residual stream in 32
        _dropout("dropout_stream", 32768, 1024, 0.1, "float", "bfloat16"),
        # gradient of rows of an odd length
        _dropout("dropout_odd_backward", 16001, 1537, 0.25, "none", "float16", backward=True),
    ]


def _spread(rng, low, high):
    return math.exp(rng.uniform(math.log(low), math.log(high)))


def draw(rng):
    op = rng.choice(["norm", "bias", "dropout"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    size = 4 if dtype == "float32" else 2
    back = rng.random() < 0.5
    moved = _spread(rng, SMALLEST, LARGEST[op])
    if op == "norm":
        groups = rng.choice([1, 3, 4, 8, 16, 32, 32])
        channels = groups * rng.choice([1, 2, 3, 4, 8, 8, 15, 16])
        values = moved / size / (3 if back else 2)
        side = min(_spread(rng, 1, 128), math.sqrt(values / channels))
        h = max(1, round(side * rng.uniform(0.75, 1.33)))
        w = max(1, round(side * side / h), math.ceil(16 * groups / (channels * h)))      # (of two values a group's gradient is nothing but roundings)
        c = _norm("", max(1, min(4096, int(values / (h * w * channels)))), (h, w), channels, groups, rng.choice(["none", "relu", "silu", "silu", "gelu"]), dtype, back)
    elif op == "bias":
        axes = rng.choice([1, 1, 2, 2, 3])
        heads = rng.choice([1, 2, 3, 4, 6, 8, 8, 12, 12, 16, 25, 32])
        packed = axes > 1 and rng.random() < 0.5
        exact = {1: rng.choice([8, 16, 33]), 2: rng.choice([7, 8, 16, 32]), 3: rng.choice([3, 5, 8])}[axes]
        coarse, far = (rng.choice([4, 8, 15]), exact * rng.choice([4, 16, 50])) if axes == 1 or (axes == 2 and rng.random() < 0.3) else (0, 0)
        pairs = moved / size / heads
        keys = max(1, int(_spread(rng, 16, 8192)))
        queries = keys if packed or back or rng.random() < 0.7 else 1
        if queries * keys > pairs:
            queries, keys = (1, int(pairs)) if queries == 1 else (int(math.sqrt(pairs)),) * 2
            queries, keys = max(1, queries), max(1, keys)
        batch = max(1, min(64, int(pairs / (queries * keys))))
        c = _bias("", batch, queries, keys, heads, axes, (exact, coarse, far), dtype, axes == 1 and rng.random() < 0.5, packed, back)
    else:
        dim = int(_spread(rng, 17, 9000)) if rng.random() < 0.4 else rng.choice([64, 192, 384, 512, 768, 1024, 2048, 4096])
        residual = "none" if back and rng.random() < 0.5 else rng.choice(["none", "same", "same", "float"])
        c = _dropout("", 1, dim, rng.choice([0.0, 0.05, 0.1, 0.1, 0.2, 0.5]), residual, dtype, back)
        c["rows"] = max(1, int(moved / work(c)["bytes"]))
    del c["name"]
    return c


# ---- inputs ----

class State:
    pass


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    S = State()
    S.case, S.dtype = case, DTYPES[case["dtype"]]
    {"norm": _prepare_norm, "bias": _prepare_bias, "dropout": _prepare_dropout}[case["op"]](S, case, _generator(seed), seed)
    return S


def _prepare_norm(S, case, gen, seed):
    N, H, W, C, G = case["images"], case["height"], case["width"], case["channels"], case["groups"]
    # feature maps: channels of different means and sizes
    mean, size = torch.randn(C, generator=gen, device="cuda"), 0.5 + torch.rand(C, generator=gen, device="cuda")
    S.x = (torch.randn((N, H, W, C), generator=gen, device="cuda") * size + mean).to(S.dtype)
    S.weight, S.bias = (1 + 0.2 * torch.randn(C, generator=gen, device="cuda")).to(S.dtype), _normal(gen, (C,), S.dtype, 0.2)
    if case["backward"]:
        S.grad = _normal(gen, (N, H, W, C), S.dtype)
        x = S.x.view(N, H * W, G, C // G).double()
        m = x.mean((1, 3))
        v = (x - m[:, None, :, None]).square().mean((1, 3))
        S.stats = torch.stack([m, (v + EPS) ** -0.5], -1).float()


def _side(case):
    """Buckets of one side of an axis, distance 0 among them."""
    return case["exact"] + case["coarse"]


def _buckets(case):
    each = _side(case) if case["one_sided"] else 2 * _side(case) - 1
    return each, each ** case["axes"]


def _map(case):
    """int32 [axes, 2 reach + 1]: what each difference (key minus query, held between -reach and reach) of an axis adds to the bucket."""
    exact, coarse, far = case["exact"], case["coarse"], case["far"]
    reach = far if coarse else exact - 1
    d = [min(x, exact - 1) if x < exact or not coarse else
         exact + max(j for j in range(coarse) if x ** coarse * exact ** j >= exact ** coarse * far ** j) for x in range(reach + 1)]
    each, _ = _buckets(case)
    if case["one_sided"]:
        row = d[:0:-1] + [0] * (reach + 1)
    else:
        row = [_side(case) - 1 - x for x in d[:0:-1]] + [_side(case) - 1 + x for x in d]
    return np.array([[v * each ** (case["axes"] - 1 - a) for v in row] for a in range(case["axes"])], np.int32)


def _places(case, tokens, rng):
    """(positions [axes, batch, tokens], segments [batch, tokens]): pictures (or clips) line by line one behind the other, or one line of tokens."""
    A, B = case["axes"], case["batch"]
    positions, segments = np.zeros((A, B, tokens), np.int32), np.full((B, tokens), -1, np.int32)
    for b in range(B):
        at = picture = 0
        while at < tokens:
            if A == 1:
                shape = (tokens,)
            elif case["packed"]:
                side = min(case["exact"] if A == 3 else 2 * case["exact"], max(2, int(tokens ** (1 / A))))
                shape = tuple(int(v) for v in rng.integers(max(1, side // 2), side + 1, size=A))
            else:
                side = math.ceil(tokens ** (1 / A))
                shape = (side,) * A
            n = math.prod(shape)
            if case["packed"] and at + n > tokens and at:
                break                                      # (what is left is padding)
            n = min(n, tokens - at)
            positions[:, b, at:at + n] = np.stack(np.unravel_index(np.arange(n), shape))
            segments[b, at:at + n] = picture
            at += n
            picture += 1
    return positions, segments


def _prepare_bias(S, case, gen, seed):
    B, Q, K, H = case["batch"], case["queries"], case["keys"], case["heads"]
    S.count = _buckets(case)[1]
    S.map = torch.from_numpy(_map(case)).cuda()
    positions, segments = _places(case, K, np.random.default_rng(seed))
    S.key_positions = torch.from_numpy(positions).cuda()
    S.key_segments = torch.from_numpy(segments).cuda() if case["packed"] else None
    S.positions, S.segments = S.key_positions, S.key_segments
    if Q != K:                                             # the newest tokens
        S.positions = S.key_positions[:, :, K - Q:].contiguous()
        S.segments = S.key_segments[:, K - Q:].contiguous() if case["packed"] else None
    if case["backward"]:
        S.grad = _normal(gen, (B, H, Q, K), S.dtype)
    else:
        S.table = _normal(gen, (S.count, H), S.dtype)


def _prepare_dropout(S, case, gen, seed):
    shape = case["rows"], case["dim"]
    S.kind = torch.float32 if case["residual"] == "float" else S.dtype        # of the result
    S.seed = torch.tensor([seed * 0x9E3779B97F4A7C15 % 2 ** 63, 1000 + seed % 1000], dtype=torch.int64, device="cuda")      # key and step
    S.call = seed % 50                                     # which of a network's dropouts
    if case["backward"]:
        S.grad = _normal(gen, shape, S.kind)
    else:
        S.x = _normal(gen, shape, S.dtype)
        S.residual = None if case["residual"] == "none" else _normal(gen, shape, S.kind, 3.0)


# ---- a pass ----

def run(S):
    return _run_own(S) if own else {"norm": _plain_norm, "bias": _plain_bias, "dropout": _plain_dropout}[S.case["op"]](S)


def _run_own(S):
    import paper_1911_00472_amd as pcr
    case = S.case
    if case["op"] == "norm":
        if case["backward"]:
            return pcr.group_norm_backward(S.grad, S.x, case["groups"], S.weight, S.bias, S.stats, activation=case["activation"])
        return pcr.group_norm_forward(S.x, case["groups"], S.weight, S.bias, eps=EPS, activation=case["activation"])
    if case["op"] == "bias":
        if case["backward"]:
            return pcr.position_bias_backward(S.grad, S.positions, S.map, S.count, key_positions=S.key_positions, segments=S.segments, key_segments=S.key_segments)
        return pcr.position_bias(S.table, S.positions, S.map, key_positions=S.key_positions, segments=S.segments, key_segments=S.key_segments)
    if case["backward"]:
        return pcr.dropout_backward(S.grad, case["p"], S.seed, call=S.call, dtype=S.dtype)
    return pcr.dropout(S.x, case["p"], S.seed, call=S.call, residual=S.residual)


def _activated(z, kind):
    """(the activation of z, its derivative)"""
    if kind == "relu":
        return torch.where(z <= 0, 0.0, z), torch.where(z <= 0, 0.0, 1.0)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if kind == "gelu":
        under = 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
        return z * under, under + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return z, torch.ones_like(z)


def _plain_norm(S):
    case = S.case
    N, C, G = case["images"], case["channels"], case["groups"]
    x = S.x.float().view(N, -1, G, C // G)
    w, b = S.weight.float().view(G, -1), S.bias.float().view(G, -1)
    if not case["backward"]:
        mean = x.mean((1, 3), keepdim=True)
        r = torch.rsqrt((x - mean).square().mean((1, 3), keepdim=True) + EPS)
        y, _ = _activated((x - mean) * r * w + b, case["activation"])
        return y.view(S.x.shape).to(S.dtype), torch.stack([mean.view(N, G), r.view(N, G)], -1)
    mean, r = S.stats[:, None, :, None, 0], S.stats[:, None, :, None, 1]
    u = (x - mean) * r
    if case["activation"] == "relu":                       # (in 64 bits: on which side of 0)
        slope = torch.where((x.double() - mean) * r * w + b <= 0, 0.0, 1.0).float()
    else:
        _, slope = _activated(u * w + b, case["activation"])
    g = S.grad.float().view(x.shape) * slope
    gw = g * w
    dx = r * (gw - gw.mean((1, 3), keepdim=True) - u * (gw * u).mean((1, 3), keepdim=True))
    return dx.view(S.x.shape).to(S.dtype), (g * u).sum((0, 1)).view(C), g.sum((0, 1)).view(C)


def _pairs(S):
    """(bucket [batch, queries, keys], whether the pair belongs together)"""
    reach = S.map.shape[1] // 2
    d = S.key_positions[:, :, None, :].long() - S.positions[:, :, :, None]
    bucket = sum(S.map[a].long()[d[a].clamp(-reach, reach) + reach] for a in range(S.map.shape[0]))
    return bucket, None if S.segments is None else S.segments[:, :, None] == S.key_segments[:, None, :]


def _plain_bias(S):
    bucket, together = _pairs(S)
    if not S.case["backward"]:
        y = S.table.float()[bucket].permute(0, 3, 1, 2)
        if together is not None:
            y = torch.where(together[:, None], y, -math.inf)
            y = torch.where((S.segments < 0)[:, None, :, None], 0.0, y)          # rows of padding
        return y.to(S.dtype, memory_format=torch.contiguous_format)
    # sums between the places where one bucket's pairs begin and end, in 64 bits
    bucket = bucket.reshape(-1)
    if together is not None:
        bucket = torch.where((together & (S.segments >= 0)[:, :, None]).view(-1), bucket, S.count)
    bucket, order = bucket.sort()
    g = S.grad.transpose(0, 1).reshape(S.case["heads"], -1)[:, order].double()
    upto = torch.cat([torch.zeros_like(g[:, :1]), g.cumsum(1)], 1)
    ends = torch.searchsorted(bucket, torch.arange(S.count + 1, device="cuda"))
    return (upto[:, ends[1:]] - upto[:, ends[:-1]]).T.float().contiguous()


def _plain_words(S, n):
    """The generator's words for n elements, in 64-bit integers of which 32 bits are used."""
    low = 0xFFFFFFFF
    group = torch.arange((n + 3) // 4, device="cuda")
    key, step = S.seed[0], S.seed[1]
    k0, k1 = key & low, (key >> 32) & low
    a, b, c, d = group & low, (group >> 32) | S.call << 16, (step & low).expand_as(group), ((step >> 32) & low).expand_as(group)
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57               # (mod 2^64: the upper half's bits are right, its sign is not looked at)
        a, b, c, d = ((q >> 32) & low) ^ b ^ k0, q & low, ((p >> 32) & low) ^ d ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([a, b, c, d], -1).view(-1)[:n]


def _plain_dropout(S):
    x = S.grad if S.case["backward"] else S.x
    p = S.case["p"]
    kept = (_plain_words(S, x.numel()) >= round(p * 2 ** 32)).view(x.shape)
    y = torch.where(kept, x.float() * (1 / (1 - p)), 0.0)
    if S.case["backward"]:
        return y.to(S.dtype)
    return (y if S.residual is None else y + S.residual.float()).to(S.kind)


# ---- the definition in 64 bits ----

def exact(case, seed):
    S = prepare(case, seed)

    def norm():
        """Group by group of channels; gradients by differentiation of the definition."""
        N, C, G = case["images"], case["channels"], case["groups"]
        x, w, b = (t.double().requires_grad_(case["backward"]) for t in (S.x, S.weight, S.bias))
        parts, stats = [], []
        for g in range(G):
            at = slice(g * C // G, (g + 1) * C // G)
            u = x[..., at]
            m = u.sum((1, 2, 3)) / u[0].numel()
            off = u - m[:, None, None, None]
            v = (off * off).sum((1, 2, 3)) / u[0].numel() + EPS
            z = off / torch.sqrt(v)[:, None, None, None] * w[at] + b[at]
            parts.append({"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z),
                          "gelu": lambda: z * torch.special.ndtr(z)}[case["activation"]]())
            stats.append(torch.stack([m, v ** -0.5], -1))
        y = torch.cat(parts, -1)
        if not case["backward"]:
            return y, torch.stack(stats, 1)
        return torch.autograd.grad((y * S.grad.double()).sum(), (x, w, b))

    def bias():
        """A row of queries at a time, buckets from the definition."""
        B, Q, H = case["batch"], case["queries"], case["heads"]
        e, coarse, far = case["exact"], case["coarse"], case["far"]
        # where the bucket of a distance changes: 1, 2 .. exact, then exact (far / exact)^(j / coarse)
        borders = [float(v) for v in range(1, e + (1 if coarse else 0))]
        borders += [next(x for x in range(e, far + 1) if x ** coarse * e ** j >= e ** coarse * far ** j) for j in range(1, coarse)]
        borders = torch.tensor(borders, dtype=torch.float64, device="cuda")
        each, count = _buckets(case)
        out = torch.empty((B, H, Q, case["keys"]), dtype=torch.float64, device="cuda") if not case["backward"] else None
        total = torch.zeros((count, H), dtype=torch.float64, device="cuda") if case["backward"] else None
        step = max(1, (1 << 24) // (B * case["keys"]))
        for i in range(0, Q, step):
            bucket = 0
            for a in range(case["axes"]):
                d = S.key_positions[a, :, None, :].double() - S.positions[a, :, i:i + step, None].double()
                if case["one_sided"]:
                    near = torch.searchsorted(borders, (-d).clamp(min=0), right=True)
                else:
                    near = _side(case) - 1 + torch.sign(d).long() * torch.searchsorted(borders, d.abs(), right=True)
                bucket = bucket * each + near
            apart = padding = None
            if case["packed"]:
                mine = S.segments[:, i:i + step, None]
                apart, padding = mine != S.key_segments[:, None], (mine < 0).expand(-1, -1, case["keys"])
            for h in range(H):
                if out is not None:
                    v = S.table[:, h].double()[bucket]
                    if apart is not None:
                        v = v.masked_fill(apart, -math.inf).masked_fill(padding, 0.0)
                    out[:, h, i:i + step] = v
                else:
                    g = S.grad[:, h, i:i + step].double()
                    if apart is not None:
                        g = g.masked_fill(apart | padding, 0.0)
                    total[:, h] += torch.bincount(bucket.reshape(-1), g.reshape(-1), minlength=count)
        return out if out is not None else total

    def dropout():
        """The generator in unsigned integers on the host."""
        x = S.grad if case["backward"] else S.x
        n, low = x.numel(), np.uint64(0xFFFFFFFF)
        key, step = (int(v) for v in S.seed.tolist())
        group = np.arange((n + 3) // 4, dtype=np.uint64)
        word = [group & low, (group >> np.uint64(32)) + np.uint64(S.call * 65536), np.full_like(group, step & 0xFFFFFFFF), np.full_like(group, step >> 32)]
        for i in range(10):
            k = [np.uint64((key + i * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((key >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)]
            first, second = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
            word = [(second >> np.uint64(32)) ^ word[1] ^ k[0], second & low, (first >> np.uint64(32)) ^ word[3] ^ k[1], first & low]
        kept = np.stack(word, 1).reshape(-1)[:n] >= np.uint64(round(case["p"] * 2 ** 32))
        y = x.double() * torch.from_numpy(kept).view(x.shape).cuda() / (1 - case["p"])
        return y if case["backward"] or S.residual is None else y + S.residual.double()

    return {"norm": norm, "bias": bias, "dropout": dropout}[case["op"]]()


# ---- what a pass cannot do without ----

def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    back = case["backward"]
    if case["op"] == "norm":
        values = float(case["images"]) * case["height"] * case["width"] * case["channels"]
        few = case["channels"] * (2 * size + (8 if back else 0)) + case["images"] * case["groups"] * 8
        return {"bytes": values * size * (3 if back else 2) + few, "flops": values * (20 if back else 12)}
    if case["op"] == "bias":
        values = float(case["batch"]) * case["heads"] * case["queries"] * case["keys"]
        tokens = case["batch"] * (case["keys"] + (case["queries"] if case["queries"] != case["keys"] else 0))
        table = _buckets(case)[1] * case["heads"] * (4 if back else size)
        return {"bytes": values * size + table + tokens * 4 * (case["axes"] + (1 if case["packed"] else 0)),
                "flops": values + 3.0 * values / case["heads"] * case["axes"]}
    values, of_result = float(case["rows"]) * case["dim"], 4 if case["residual"] == "float" else size
    moved = size + of_result * (2 if case["residual"] != "none" and not back else 1)
    return {"bytes": values * moved + 16, "flops": values * 3}

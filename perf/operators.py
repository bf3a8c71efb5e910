"""The operators between a decoded record and a transformer that trains on it: what is timed, in a plain form and through the package.

A record's pictures (ragged uint8 pixels, image after image) become patch rows with positions; queries and keys are normalised and
rotated by those positions (time, row, column); a student that sees a low scan group learns from the top logits of a teacher that saw
the full one.  A case is a dict of plain values:

  op        patch     pixels to normalised patch rows and their positions
            rotate    positions of several axes turned into queries and keys; `inverse`: its gradient
            norm      the same behind a norm of every head; `backward`: its gradient
            distill   loss against a teacher's top logits, beside the labels' where `labels` is true; `mode`: forward (loss), backward
                      (gradient from the saved sums), step (both in one pass)
  dtype     of what is read and written
  patch:        images, w0..w1, h0..h1 (sides drawn uniformly), channels, patch (side), merge (patches that follow each other), frames
  rotate, norm: batch, tokens (of one sequence), qheads, kheads, dim, pairs (rotated pairs of a head), axes, adjacent (pairs of neighbours
                instead of halves), memory (split: tensors of their own; fused: views of one projection's output; heads: heads before tokens),
                far (positions below it)
  distill:      rows, classes, top, temperature
"""
import math

import numpy as np
import torch

own = False

MEAN, INV_STD = (0.485, 0.456, 0.406), (1 / 0.229, 1 / 0.224, 1 / 0.225)
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
LARGEST = 2.0e9                                          # bytes that a drawn case moves at most
SMALLEST = 1.0e4


def _patch(name, images, size, patch, dtype, channels=3, merge=1, frames=1):
    return {"name": name, "op": "patch", "images": images, "w0": size[0], "w1": size[1], "h0": size[2], "h1": size[3], "channels": channels,
            "patch": patch, "merge": merge, "frames": frames, "dtype": dtype}


def _heads(name, op, batch, tokens, qheads, kheads, dim, pairs, axes, dtype, adjacent=False, memory="split", far=4096, back=False):
    c = {"name": name, "op": op, "batch": batch, "tokens": tokens, "qheads": qheads, "kheads": kheads, "dim": dim, "pairs": pairs, "axes": axes,
         "adjacent": adjacent, "memory": memory, "far": far, "dtype": dtype}
    c["inverse" if op == "rotate" else "backward"] = back
    return c


def _distill(name, mode, rows, classes, top, dtype, temperature=1.0, labels=False):
    return {"name": name, "op": "distill", "mode": mode, "rows": rows, "classes": classes, "top": top, "temperature": temperature, "labels": labels,
            "dtype": dtype}


def listed():
    return [
        # a handful of gray thumbnails: launches and latency
        _patch("patch_gray64", 64, (64, 64, 64, 64), 8, "float16", channels=1),
        # a record of photographs of 300 to 500 pixels at their own sizes, patches of a window after each other
        _patch("patch_photos", 1024, (300, 500, 300, 500), 14, "bfloat16", merge=2),
        # one new token of 32 sequences that are being answered at once
        _heads("rotate_token", "rotate", 32, 1, 32, 8, 128, 64, 3, "bfloat16", far=32768),
        # the patches of a batch of pictures in an encoder, queries and keys inside a fused projection's output
        _heads("rotate_pictures", "rotate", 1, 49999, 16, 16, 72, 36, 2, "float16", adjacent=True, memory="fused", far=64),
        # gradient of long clips
        _heads("rotate_clips_inverse", "rotate", 2, 32768, 32, 8, 128, 64, 3, "bfloat16", far=4096, back=True),
        # a single token of a single sequence
        _heads("norm_token", "norm", 1, 1, 32, 8, 128, 64, 3, "bfloat16", far=32768),
        # prompts with pictures in 32 bits, a third of each head left as it is, heads before tokens
        _heads("norm_prompt", "norm", 4, 2051, 12, 4, 96, 32, 3, "float32", memory="heads", far=1024),
        # gradient in a training step
        _heads("norm_train_backward", "norm", 8, 4096, 32, 8, 128, 64, 3, "bfloat16", memory="fused", far=4096, back=True),
        # a classifier of a thousand classes learning from ten of the teacher's logits and the labels
        _distill("distill_classes", "step", 1024, 1000, 10, "float32", 2.0, True),
        # the loss of a few rows over a long vocabulary
        _distill("distill_few_rows", "forward", 7, 131071, 64, "bfloat16"),
        # a training step over an odd vocabulary, labels beside
        _distill("distill_tokens", "step", 4096, 50001, 32, "bfloat16", 2.0, True),
        # the gradient from the saved sums over a long vocabulary
        _distill("distill_long_backward", "backward", 4096, 131072, 128, "float16", 1.5),
    ]


def _spread(rng, low, high):
    return math.exp(rng.uniform(math.log(low), math.log(high)))


def draw(rng):
    op = rng.choice(["patch", "rotate", "norm", "distill"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    size = 4 if dtype == "float32" else 2
    moved = _spread(rng, SMALLEST, LARGEST)
    if op == "patch":
        side = _spread(rng, 24, 1024)
        w = max(9, round(side * rng.uniform(0.75, 1.33)))
        h = max(9, round(side * side / w))
        spread = rng.choice([1.0, 1.3, 1.6])
        channels = rng.choice([3, 3, 3, 1])
        c = _patch("", 1, (int(w / spread), int(w * spread), int(h / spread), int(h * spread)), rng.choice([8, 14, 16, 20, 28]), dtype, channels,
                   rng.choice([1, 1, 2]), rng.choice([1, 1, 4, 16]))
        c["images"] = max(1, min(4096, int(moved / 2 / work(c)["bytes"])))
    elif op == "distill":
        classes = int(_spread(rng, 100, 160000))
        mode = rng.choice(["forward", "backward", "step"])
        rows = max(1, min(16384, int(moved / (classes * size * (1 if mode == "forward" else 2)))))
        c = _distill("", mode, rows, classes, min(classes, rng.choice([1, 5, 10, 32, 50, 64, 100, 128, 256])), dtype,
                     rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]), rng.random() < 0.5)
    else:
        dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 256])
        qheads = rng.choice([1, 2, 7, 9, 13, 17, 28, 40])
        kheads = rng.choice([qheads, max(1, qheads // 4), max(1, qheads // 8)])
        axes = rng.choice([1, 2, 3, 3])
        pairs = dim // 2 if rng.random() < 0.75 else dim // 4
        back = rng.random() < 0.5
        tokens = max(1, int(moved / ((3 if op == "norm" and back else 2) * (qheads + kheads) * dim * size)))
        batch = min(tokens, rng.choice([1, 1, 2, 8, 32]))
        c = _heads("", op, batch, tokens // batch, qheads, kheads, dim, pairs, axes, dtype, rng.random() < 0.3, rng.choice(["split", "fused", "heads"]),
                   rng.choice([32, 256, 1024]) if dtype == "float32" else rng.choice([64, 1024, 32768]), back)
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
    S.case = case
    gen = _generator(seed)
    {"patch": _prepare_patch, "rotate": _prepare_heads, "norm": _prepare_heads, "distill": _prepare_distill}[case["op"]](S, case, gen)
    return S


def _sides(case):
    """(heights, widths) of the pictures: they belong to the case, what the pictures show to the seed."""
    rng = np.random.default_rng(191100472)
    W = rng.integers(case["w0"], case["w1"] + 1, size=case["images"])
    H = rng.integers(case["h0"], case["h1"] + 1, size=case["images"])
    return H.astype(np.int64), W.astype(np.int64)


def _grid(case):
    H, W = _sides(case)
    cell = case["patch"] * case["merge"]
    return -(-H // cell) * case["merge"], -(-W // cell) * case["merge"]


def _prepare_patch(S, case, gen):
    H, W = _sides(case)
    rows, columns = _grid(case)
    offsets = np.concatenate([[0], np.cumsum(H * W * case["channels"])])
    first = np.concatenate([[0], np.cumsum(rows * columns)])
    S.rows = int(first[-1])
    S.shapes = torch.from_numpy(np.stack([H, W], 1).astype(np.int32)).cuda()
    S.offsets = torch.from_numpy(offsets).cuda()
    S.first = torch.from_numpy(first).cuda()
    S.mean, S.inv_std = MEAN[:case["channels"]], INV_STD[:case["channels"]]
    S.pixels = torch.randint(0, 256, (int(offsets[-1]),), generator=gen, device="cuda", dtype=torch.uint8)


def _prepare_heads(S, case, gen):
    B, T, Hq, Hk, D, A = case["batch"], case["tokens"], case["qheads"], case["kheads"], case["dim"], case["axes"]
    dtype, pairs = DTYPES[case["dtype"]], case["pairs"]

    def tensors():
        if case["memory"] == "fused":                  # queries, keys and values of a token side by side
            x = _normal(gen, (B, T, (Hq + 2 * Hk) * D), dtype)
            return x[..., :Hq * D].unflatten(-1, (Hq, D)), x[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D))
        if case["memory"] == "heads":
            return _normal(gen, (B, Hq, T, D), dtype).transpose(1, 2), _normal(gen, (B, Hk, T, D), dtype).transpose(1, 2)
        return _normal(gen, (B, T, Hq, D), dtype), _normal(gen, (B, T, Hk, D), dtype)

    S.q, S.k = tensors()
    S.positions = torch.randint(0, case["far"], (A, B, T), generator=gen, device="cuda", dtype=torch.int32)
    each = [pairs // A] * (A - 1)
    each.append(pairs - sum(each))                     # pairs of every axis, one axis after another
    S.axis = torch.repeat_interleave(torch.arange(A), torch.tensor(each)).to(device="cuda", dtype=torch.int32)
    if A == 2:                                         # rows and columns: each its own run of frequencies
        power = torch.cat([torch.arange(n, dtype=torch.float64) / max(n, 1) for n in each])
    else:                                              # one run over all pairs
        power = torch.arange(pairs, dtype=torch.float64) / max(pairs, 1)
    S.frequency = (10000.0 ** -power).to(device="cuda", dtype=torch.float32)
    S.eps = 1e-6
    if case["op"] == "norm":
        S.qweight, S.kweight = ((1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(dtype) for _ in range(2))
        if case["backward"]:
            S.gq, S.gk = _normal(gen, (B, T, Hq, D), dtype), _normal(gen, (B, T, Hk, D), dtype)


def _prepare_distill(S, case, gen):
    N, V, K = case["rows"], case["classes"], case["top"]
    dtype = DTYPES[case["dtype"]]
    S.logits = _normal(gen, (N, V), dtype, 1.5)
    # entries of a row: distinct classes spread over the vocabulary, the teacher's logits falling from the first on
    start = torch.randint(0, V, (N, 1), generator=gen, device="cuda")
    step = V // K
    jitter = torch.randint(0, max(step, 1), (N, K), generator=gen, device="cuda")
    S.top_index = (start + torch.arange(K, device="cuda") * step + jitter) % V
    S.top_logits = (8 - 1.2 * torch.arange(K, device="cuda").add(1).log() * (1 + torch.rand((N, 1), generator=gen, device="cuda"))
                    + 0.2 * torch.randn((N, K), generator=gen, device="cuda")).to(dtype)
    S.logits.scatter_(1, S.top_index, (S.top_logits.float() + torch.randn((N, K), generator=gen, device="cuda")).to(dtype))
    gone = torch.rand((N, K), generator=gen, device="cuda") < 0.02
    S.top_index = S.top_index.masked_fill_(gone, -1).to(torch.int32)      # a teacher that kept fewer
    S.labels = None
    if case["labels"]:
        S.labels = torch.randint(0, V, (N,), generator=gen, device="cuda")
        S.labels.masked_fill_(torch.rand(N, generator=gen, device="cuda") < 0.05, -100)
    S.part = (0.7, 0.3) if case["labels"] else (1.0, 0.0)
    scale = 65536.0 if dtype == torch.float16 else 1.0         # (a loss is scaled up where its gradient is held in half precision)
    S.weight = torch.rand(N, generator=gen, device="cuda") * (scale / N)
    S.weight.masked_fill_(torch.rand(N, generator=gen, device="cuda") < 0.03, 0.0)             # rows of padding
    if case["mode"] == "backward":
        S.sums = torch.zeros((N, 2), dtype=torch.float32, device="cuda")
        S.sums[:, 0] = torch.logsumexp(S.logits.double() / case["temperature"], 1)
        if case["labels"]:
            S.sums[:, 1] = torch.logsumexp(S.logits.double(), 1)


# ---- a pass ----

def run(S):
    return _run_own(S) if own else {"patch": _plain_patch, "rotate": _plain_rotate, "norm": _plain_norm, "distill": _plain_distill}[S.case["op"]](S)


def _run_own(S):
    import paper_1911_00472_amd as pcr
    case = S.case
    op = case["op"]
    if op == "patch":
        return pcr.patch_rows(S.pixels, S.shapes, S.offsets, S.first, S.rows, case["patch"], S.mean, S.inv_std, merge=case["merge"], frames=case["frames"],
                              dtype=DTYPES[case["dtype"]])
    if op == "rotate":
        return pcr.rotate_axes(S.q, S.k, S.positions, S.frequency, S.axis, adjacent=case["adjacent"], inverse=case["inverse"])
    if op == "norm":
        if case["backward"]:
            return pcr.norm_rotate_backward(S.gq, S.gk, S.q, S.k, S.qweight, S.kweight, S.positions, S.frequency, S.axis, eps=S.eps,
                                            adjacent=case["adjacent"])
        return pcr.norm_rotate(S.q, S.k, S.qweight, S.kweight, S.positions, S.frequency, S.axis, eps=S.eps, adjacent=case["adjacent"])
    a, b = S.part
    more = {"labels": S.labels, "temperature": case["temperature"], "distill_part": a, "label_part": b}
    if case["mode"] == "forward":
        return pcr.distill_forward(S.logits, S.top_index, S.top_logits, **more)
    if case["mode"] == "backward":
        return pcr.distill_backward(S.weight, S.logits, S.top_index, S.top_logits, S.sums, **more)
    return pcr.distill_step(S.logits, S.top_index, S.top_logits, S.weight, **more)


def _plain_patch(S):
    case = S.case
    P, C, m = case["patch"], case["channels"], case["merge"]
    cell = P * m
    token = torch.arange(S.rows, device="cuda")
    image = torch.searchsorted(S.first, token, right=True) - 1
    height, width = S.shapes[image, 0].long(), S.shapes[image, 1].long()
    place = token - S.first[image]
    window, inside = place // (m * m), place % (m * m)
    across = (width + cell - 1) // cell
    row, column = window // across * m + inside // m, window % across * m + inside % m
    positions = torch.stack([image % case["frames"], row, column]).to(torch.int32)
    reach = torch.arange(P, device="cuda")
    y, x = (row[:, None] * P + reach)[:, None, :, None], (column[:, None] * P + reach)[:, None, None, :]
    there = (y < height[:, None, None, None]) & (x < width[:, None, None, None])
    at = S.offsets[image][:, None, None, None] + (y * width[:, None, None, None] + x) * C + torch.arange(C, device="cuda")[:, None, None]
    value = S.pixels[torch.where(there, at, 0)].float()
    mean = torch.tensor(S.mean, device="cuda")[:, None, None]
    inv_std = torch.tensor(S.inv_std, device="cuda")[:, None, None]
    value = torch.where(there, (value / 255 - mean) * inv_std, 0.0)
    return value.reshape(S.rows, C * P * P).to(DTYPES[case["dtype"]]), positions


def _turn(x, S, sign):
    """x [batch, tokens, heads, dim] in 32 bits, its pairs turned by the positions' angles."""
    n = S.case["pairs"]
    angle = (S.positions[S.axis.long()].float() * S.frequency[:, None, None]).permute(1, 2, 0)[:, :, None]
    c, s = torch.cos(angle), torch.sin(angle) * sign
    if S.case["adjacent"]:
        u, v = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack([u * c - v * s, u * s + v * c], -1).flatten(-2)
    else:
        u, v = x[..., :n], x[..., n:2 * n]
        turned = torch.cat([u * c - v * s, u * s + v * c], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_rotate(S):
    dtype, sign = DTYPES[S.case["dtype"]], -1.0 if S.case["inverse"] else 1.0
    return _turn(S.q.float(), S, sign).to(dtype), _turn(S.k.float(), S, sign).to(dtype)


def _plain_norm(S):
    dtype = DTYPES[S.case["dtype"]]

    def forward(x, w):
        x = x.float()
        return _turn(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + S.eps) * w.float(), S, 1.0).to(dtype)

    def backward(g, x, w):
        x, g = x.float(), _turn(g.float(), S, -1.0)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + S.eps)
        gw = g * w.float()
        dx = r * (gw - x * (r * r) * (gw * x).mean(-1, keepdim=True))
        return dx.to(dtype), (g * x * r).sum((0, 1, 2))

    if S.case["backward"]:
        (dq, dqw), (dk, dkw) = backward(S.gq, S.q, S.qweight), backward(S.gk, S.k, S.kweight)
        return dq, dk, dqw, dkw
    return forward(S.q, S.qweight), forward(S.k, S.kweight)


def _plain_distill(S):
    case = S.case
    V, temperature, mode = case["classes"], case["temperature"], case["mode"]
    a, b = S.part
    z = S.logits.float()
    valid = (S.top_index >= 0) & (S.top_index < V)
    index = torch.where(valid, S.top_index, 0).long()
    t = torch.where(valid, S.top_logits.float() / temperature, -math.inf)
    t = t - t.max(1, keepdim=True).values.clamp(min=-1e30)
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    p = torch.where(valid, e / total.clamp(min=1e-30), 0.0)
    labelled = S.labels is not None and b != 0
    if labelled:
        counted = (S.labels >= 0) & (S.labels < V)
        label = torch.where(counted, S.labels, 0)[:, None]
    if mode == "backward":
        lse, lse1 = S.sums[:, :1], S.sums[:, 1:]
    else:
        most = z.max(1, keepdim=True).values
        lse = torch.log(torch.exp((z - most) / temperature).sum(1, keepdim=True)) + most / temperature
        lse1 = torch.log(torch.exp(z - most).sum(1, keepdim=True)) + most if labelled else torch.zeros_like(lse)
        log_p = torch.where(valid, t - torch.log(total), 0.0)
        loss = a * temperature ** 2 * (p * (log_p - (z.gather(1, index) / temperature - lse))).sum(1)
        if labelled:
            loss = loss + b * torch.where(counted, (lse1 - z.gather(1, label))[:, 0], 0.0)
        if mode == "forward":
            return loss, torch.cat([lse, lse1], 1)
    grad = torch.exp(z / temperature - lse) * p.sum(1, keepdim=True)
    grad.scatter_add_(1, index, -p)
    grad = grad * (a * temperature)
    if labelled:
        by_label = torch.exp(z - lse1)
        by_label.scatter_add_(1, label, torch.full_like(lse, -1.0))
        grad = grad + torch.where(counted[:, None], by_label * b, 0.0)
    grad = (grad * S.weight[:, None]).to(DTYPES[case["dtype"]])
    return grad if mode == "backward" else (loss * S.weight, grad)


# ---- the definition in 64 bits ----

def exact(case, seed):
    S = prepare(case, seed)

    def patch():
        """Picture by picture: padded, cut by folding its axes."""
        P, C, m = case["patch"], case["channels"], case["merge"]
        cell = P * m
        H, W = _sides(case)
        mean = torch.tensor(S.mean, dtype=torch.float64, device="cuda")
        inv_std = torch.tensor(S.inv_std, dtype=torch.float64, device="cuda")
        values = torch.empty((S.rows, C * P * P), dtype=torch.float64, device="cuda")
        places = torch.empty((3, S.rows), dtype=torch.int32, device="cuda")
        done = begin = 0
        for i, (h, w) in enumerate(zip(H.tolist(), W.tolist())):
            down, across = -(-h // cell), -(-w // cell)
            picture = S.pixels[begin:begin + h * w * C].view(h, w, C).double()
            begin += h * w * C
            full = torch.zeros((down * cell, across * cell, C), dtype=torch.float64, device="cuda")
            full[:h, :w] = (picture / 255 - mean) * inv_std
            n = down * across * m * m
            values[done:done + n] = full.view(down, m, P, across, m, P, C).permute(0, 3, 1, 4, 6, 2, 5).reshape(n, C * P * P)
            rows = torch.arange(down * m, dtype=torch.int32, device="cuda").view(down, m, 1, 1).expand(-1, -1, across, m)
            columns = torch.arange(across * m, dtype=torch.int32, device="cuda").view(1, 1, across, m).expand(down, m, -1, -1)
            places[0, done:done + n] = i % case["frames"]
            places[1, done:done + n] = rows.permute(0, 2, 1, 3).reshape(-1)
            places[2, done:done + n] = columns.permute(0, 2, 1, 3).reshape(-1)
            done += n
        return values, places

    def heads():
        """Pairs as complex numbers; the norm's gradient from the projection that the norm's derivative is."""
        n, D = case["pairs"], case["dim"]
        angle = torch.stack([S.positions[int(a)].double() * float(f) for a, f in zip(S.axis.tolist(), S.frequency.double().tolist())], -1)[:, :, None]

        def turn(x, sign):
            if case["adjacent"]:
                z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous())
            else:
                z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous())
            z = z * torch.polar(torch.ones_like(angle), sign * angle)
            y = x.clone()
            if case["adjacent"]:
                y[..., :2 * n] = torch.view_as_real(z).flatten(-2)
            else:
                y[..., :n], y[..., n:2 * n] = z.real, z.imag
            return y

        if case["op"] == "rotate":
            sign = -1.0 if case["inverse"] else 1.0
            return turn(S.q.double(), sign), turn(S.k.double(), sign)

        def length(x):
            return torch.sqrt((x * x).sum(-1, keepdim=True) / D + S.eps)

        if not case["backward"]:
            return tuple(turn(x.double() / length(x.double()) * w.double(), 1.0) for x, w in ((S.q, S.qweight), (S.k, S.kweight)))
        found = []
        for g, x, w in ((S.gq, S.q, S.qweight), (S.gk, S.k, S.kweight)):
            g, x = turn(g.double(), -1.0), x.double()
            root = length(x)
            unit = x / root
            along = g * w.double()
            found.append(((along - unit * ((along * unit).sum(-1, keepdim=True) / D)) / root, (g * unit).sum((0, 1, 2))))
        return found[0][0], found[1][0], found[0][1], found[1][1]

    def distill():
        """A block of rows at a time, from log-probabilities."""
        N, V, T, mode = case["rows"], case["classes"], case["temperature"], case["mode"]
        a, b = S.part
        block = max(1, min(N, (1 << 28) // V))
        losses = torch.zeros(N, dtype=torch.float64, device="cuda")
        sums = torch.zeros((N, 2), dtype=torch.float64, device="cuda")
        grads = torch.zeros((N, V), dtype=torch.float64, device="cuda") if mode != "forward" else None
        for i in range(0, N, block):
            rows = slice(i, i + block)
            z, index, t = S.logits[rows].double(), S.top_index[rows].long(), S.top_logits[rows].double()
            kept = (index >= 0).double()
            weight = kept * torch.softmax(torch.where(kept > 0, t / T, -1e300), 1)
            teacher = torch.zeros_like(z).scatter_add_(1, index.clamp(min=0), weight)
            log_q = torch.log_softmax(z / T, 1)
            sums[rows, 0] = z[:, 0] / T - log_q[:, 0]
            loss = a * T * T * (torch.xlogy(teacher, teacher) - teacher * log_q).sum(1)
            grad = a * T * (torch.exp(log_q) * teacher.sum(1, keepdim=True) - teacher) if grads is not None else None
            if S.labels is not None:
                there = (S.labels[rows] >= 0).double()
                log_q = torch.log_softmax(z, 1)
                sums[rows, 1] = z[:, 0] - log_q[:, 0]
                at = S.labels[rows].clamp(min=0)[:, None]
                loss = loss - b * there * log_q.gather(1, at)[:, 0]
                if grads is not None:
                    grad += b * there[:, None] * torch.exp(log_q).scatter_add_(1, at, torch.full_like(there[:, None], -1.0))
            losses[rows] = loss
            if grads is not None:
                grads[rows] = grad * S.weight[rows].double()[:, None]
        if mode == "forward":
            return losses, sums
        return grads if mode == "backward" else (losses * S.weight.double(), grads)

    return {"patch": patch, "rotate": heads, "norm": heads, "distill": distill}[case["op"]]()


# ---- what a pass cannot do without ----

def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "patch":
        H, W = _sides(case)
        rows, columns = _grid(case)
        written = float((rows * columns).sum()) * case["channels"] * case["patch"] ** 2
        pixels = float((H * W).sum()) * case["channels"]
        return {"bytes": pixels + written * size + 12.0 * float((rows * columns).sum()), "flops": 2 * pixels}
    if case["op"] == "distill":
        values, K = float(case["rows"]) * case["classes"], case["top"]
        moved = values * size * (1 if case["mode"] == "forward" else 2) + case["rows"] * (K * (4 + size) + 16)
        exps = 2 if case["labels"] and case["temperature"] != 1 else 1
        return {"bytes": moved, "flops": values * 4 * exps * (1 if case["mode"] != "step" else 2)}
    tokens = float(case["batch"]) * case["tokens"]
    values = tokens * (case["qheads"] + case["kheads"]) * case["dim"]
    back = case["op"] == "norm" and case["backward"]
    flops = 3 * values * 2 * case["pairs"] / case["dim"]
    if case["op"] == "norm":
        flops += values * (12 if back else 4)
    return {"bytes": values * size * (3 if back else 2) + tokens * case["axes"] * 4, "flops": flops}

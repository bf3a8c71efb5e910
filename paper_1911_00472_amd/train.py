"""The operators between a decoded record and a transformer that trains on it (include/pcr.h): patch rows and their positions, positions
of several axes turned into queries and keys (alone or behind a norm of every head), and distillation from a teacher's top logits; and layers of a network that
trains on the pictures: group norm with an activation, a bias of attention for relative positions, dropout.

The work is done by the library's HIP kernels, enqueued on the current stream (or `stream`, a hipStream_t as an integer); arguments are checked and handed on
by the native module _train (csrc/pcr_bind.cpp).  A tensor on another stream than the one it was made on needs the caller's
record_stream, as with any operator.  Wrong types, shapes or devices raise ValueError before anything is enqueued, what the library
refuses raises PcrError.  rotate_axes, norm_rotate, distill_loss, group_norm, position_bias and dropout take part in automatic differentiation; a gradient is made on the
stream of its forward pass.  There are no derivatives of forward mode (ValueError), and no traces (RuntimeError)."""
import math
import os
from decimal import Decimal, localcontext

import numpy as np
import torch

from .binding import PcrError, lib

lib()                                                      # (the module below is linked with it)
if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_train.so")):
    raise RuntimeError("_train.so is missing: run `python -c 'import __graft_entry__ as g; g.build()'` first; there is no fallback path")
from . import _train  # noqa: E402

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_train.set_up(PcrError, getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream))


def _call(stream, f, *args):
    """f on the current stream; on `stream`, results and working memory come from that stream's pool, so that they are not handed out while it works on them."""
    if stream is None:
        return f(*args)
    index = next((a.get_device() for a in args if isinstance(a, torch.Tensor) and a.is_cuda), None)
    if index is None:                                      # (it has no tensor to work on, and says so)
        return f(*args)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=index) if stream else torch.cuda.default_stream(index)):
        return f(*args)


# ---- patch rows ----

def patch_layout(shapes, channels, patch, merge=1, offsets=None, device=0):
    """What patch_rows needs to know of pictures of the given (height, width), one behind the other as decode_batch writes them (offsets: where
    each begins, and the end): (shapes int32 [n, 2], offsets int64 [n + 1], first_rows int64 [n + 1]) as CUDA tensors, and the number of rows.
    shapes keeps the pictures' channels (an attribute of that name), which patch_rows holds against the number of means; with offsets they may be None,
    for pictures of which they are not known."""
    hw = np.asarray(shapes, np.int64).reshape(-1, 2)
    cell = patch * merge
    rows = np.where((hw > 0).all(1), (-(-hw // cell) * merge).prod(1), 0)
    if offsets is None:
        offsets = np.concatenate([[0], np.cumsum(hw.prod(1) * channels)])
    first = np.concatenate([[0], np.cumsum(rows)])
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    shapes = torch.from_numpy(hw.astype(np.int32)).to(dev)
    if channels is not None:
        shapes.channels = channels
    return shapes, torch.from_numpy(np.asarray(offsets).astype(np.int64)).to(dev), torch.from_numpy(first.astype(np.int64)).to(dev), int(first[-1])


def patch_rows(pixels, shapes, offsets, first_rows, rows, patch, mean, inv_std, merge=1, frames=1, dtype=torch.bfloat16, out=None, positions=None,
               stream=None):
    """Normalised patch rows of ragged uint8 pictures (decode_batch's pixels; shapes, offsets and first_rows from patch_layout), and their
    positions: (dtype [rows, channels * patch * patch], int32 [3, rows]: frame, row, column).  channels = len(mean), 1 or 3; see
    pcr_patch_rows for the order of the rows and for merge and frames."""
    mean = tuple(mean)
    if getattr(shapes, "channels", len(mean)) != len(mean):
        raise ValueError("mean and inv_std: a value for each of the pictures' %d channels is wanted" % shapes.channels)
    return _call(stream, _train.patch_rows, pixels, shapes, offsets, first_rows, rows, patch, mean, tuple(inv_std), merge, frames, _TYPES.get(dtype, -1), out, positions)


# ---- positions in queries and keys ----

def axis_frequencies(sections, theta=10000.0, each=False, device=0):
    """(frequency float32 [pairs], axis int32 [pairs]) for pairs that go to the axes in runs: sections[a] of them to axis a.  Pair j of n turns by
    theta^(-j / n) radians a position; each: every axis has such a run of its own instead of its part of one run over all pairs."""
    n = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    if each:
        power = np.concatenate([np.arange(m) / max(m, 1) for m in sections])
    else:
        power = np.arange(n) / max(n, 1)
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    return torch.from_numpy((theta ** -power).astype(np.float32)).to(dev), torch.from_numpy(axis.astype(np.int32)).to(dev)


class _RotateAxes(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, frequency, axis, adjacent, inverse):
        ctx.save_for_backward(positions, frequency, axis)
        ctx.how = adjacent, inverse, k is not None
        return _train.rotate_axes(q, k, positions, frequency, axis, adjacent, inverse, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        adjacent, inverse, keys = ctx.how
        gq, gk = _dense(gq), _dense(gk) if keys else None
        dq, dk = _train.rotate_axes(gq, gk, *ctx.saved_tensors, adjacent, not inverse, None, None)
        return dq, dk, None, None, None, None, None


def _dense(g):
    """A gradient as a broadcast view may come with strides of 0, which is read as it is; only a head's elements have to follow each other."""
    return g if g.stride(-1) == 1 or g.shape[-1] == 1 else g.contiguous()


def rotate_axes(q, k, positions, frequency, axis, adjacent=False, inverse=False, q_out=None, k_out=None, stream=None):
    """Turns the pairs of queries and keys by positions of up to four axes: pair j of a token's heads by positions[axis[j]] * frequency[j] radians.
    q, k: [tokens, heads, dim] or [batch, tokens, heads, dim] (k may be None) with any strides of batch, tokens and heads; positions: integers [axes,
    tokens] or [axes, batch, tokens].  A pair is (j, j + pairs), or (2 j, 2 j + 1) if `adjacent`; what is behind the pairs is not turned.  inverse:
    by minus the angle, which is the gradient.  q_out, k_out: where to (the inputs themselves, too); given, they keep the call out of automatic
    differentiation (a leaf that requires a gradient is refused, as by an operator in place).  Returns (q, k) turned."""
    if q_out is None and k_out is None and torch.is_grad_enabled() and (getattr(q, "requires_grad", False) or getattr(k, "requires_grad", False)):
        return _call(stream, _RotateAxes.apply, q, k, positions, frequency, axis, adjacent, inverse)
    return _call(stream, _train.rotate_axes, q, k, positions, frequency, axis, adjacent, inverse, q_out, k_out)


def norm_rotate_backward(gq, gk, q, k, q_weight, k_weight, positions, frequency, axis, eps=1e-6, adjacent=False, dq=None, dk=None, stream=None):
    """Gradient of norm_rotate: (dq, dk, dq_weight, dk_weight), the weights' in float32 (None where there is no weight), summed in a fixed order.  gq and gk: the
    gradients of its results; dq and dk: where to (gq and gk, or q and k, themselves, too)."""
    return _call(stream, _train.norm_rotate_backward, gq, gk, q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, dq, dk)


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, frequency, axis)
        ctx.how = eps, adjacent
        return _train.norm_rotate(q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        q, k, q_weight, k_weight, positions, frequency, axis = ctx.saved_tensors
        dq, dk, dqw, dkw = norm_rotate_backward(_dense(gq), _dense(gk) if k is not None else None, q, k, q_weight, k_weight, positions, frequency, axis, *ctx.how)
        return (dq, dk, dqw.to(q_weight.dtype) if dqw is not None else None, dkw.to(k_weight.dtype) if dkw is not None else None) + (None,) * 5


def norm_rotate(q, k, q_weight, k_weight, positions, frequency, axis, eps=1e-6, adjacent=False, q_out=None, k_out=None, stream=None):
    """rotate_axes of x * weight / sqrt(mean x^2 + eps), the mean over each head of queries and keys, in one pass and with one rounding.  Weights: [dim]
    of float32 or of the heads' type, or None.  Returns (q, k)."""
    if q_out is None and k_out is None and torch.is_grad_enabled() and (getattr(q, "requires_grad", False) or getattr(k, "requires_grad", False) or
                                                                       getattr(q_weight, "requires_grad", False) or getattr(k_weight, "requires_grad", False)):
        return _call(stream, _NormRotate.apply, q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent)
    return _call(stream, _train.norm_rotate, q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, q_out, k_out)


# ---- distillation ----

def distill_forward(logits, top_index, top_logits, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, stream=None):
    """(loss float32 [rows], sums float32 [rows, 2]): of every row distill_part * temperature^2 * the divergence of softmax(logits / temperature) from the
    softmax of the teacher's kept logits (top_logits / temperature at classes top_index; a class outside 0 .. classes - 1 does not count), and label_part
    * the cross entropy with labels (int64; one outside the classes does not count).  sums is what distill_backward takes."""
    return _call(stream, _train.distill_forward, logits, top_index, top_logits, labels, temperature, distill_part, label_part)


def distill_backward(row_grad, logits, top_index, top_logits, sums, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, out=None, stream=None):
    """The gradient of the logits for row_grad, the gradient of every row's loss (float32 [rows]), from distill_forward's sums (which are made anew from the
    logits for rows whose sums are 128 or more in magnitude).  out: where to (the logits themselves, too, if they are no leaf that requires a gradient)."""
    return _call(stream, _train.distill_backward, row_grad, logits, top_index, top_logits, sums, labels, temperature, distill_part, label_part, out)


def distill_step(logits, top_index, top_logits, row_weight, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, out=None, stream=None):
    """(loss, gradient) in one pass: loss[n] = row_weight[n] * distill_forward's loss, and the gradient of their sum.  A row of weight 0 is left out whatever
    it holds.  out: where the gradient goes (the logits themselves, too, if they are no leaf that requires a gradient)."""
    return _call(stream, _train.distill_step, logits, top_index, top_logits, row_weight, labels, temperature, distill_part, label_part, out)


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_index, top_logits, labels, temperature, distill_part, label_part):
        loss, sums = distill_forward(logits, top_index, top_logits, labels, temperature, distill_part, label_part)
        ctx.save_for_backward(logits, top_index, top_logits, sums, labels)
        ctx.how = temperature, distill_part, label_part
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        logits, top_index, top_logits, sums, labels = ctx.saved_tensors
        return (distill_backward(g.contiguous(), logits, top_index, top_logits, sums, labels, *ctx.how),) + (None,) * 6


def distill_loss(logits, top_index, top_logits, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0):
    """distill_forward's loss of every row (float32 [rows]), differentiable in the logits."""
    return _DistillLoss.apply(logits, top_index, top_logits, labels, temperature, distill_part, label_part)


# ---- group norm ----

_ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _activation(name):
    if not isinstance(name, (str, type(None))) or name not in _ACTIVATIONS:
        raise ValueError("activation: none, relu, silu or gelu is wanted")
    return _ACTIVATIONS[name]


def group_norm_forward(x, groups, weight=None, bias=None, eps=1e-5, activation=None, out=None, stream=None):
    """(y, stats) of feature maps x [images, ..., channels], channels last: activation((x - m) * weight / sqrt(var + eps) + bias), mean m and variance over the
    pixels of an image and the channels of a group.  Weight and bias: [channels] of float32 or of x's type, or None.  activation: None, "relu", "silu" or "gelu" (with the
    error function).  Pixels of any one stride (a slice of channels, too); a tensor [images, channels, height, width] in channels-last memory comes as x.permute(0, 2, 3, 1).
    stats: float32 [images, groups, 2], m and 1 / sqrt(var + eps), which group_norm_backward takes.  out: where y goes (x itself, too)."""
    return _call(stream, _train.group_norm_forward, x, groups, weight, bias, eps, _activation(activation), out)


def group_norm_backward(grad, x, groups, weight, bias, stats, activation=None, dx=None, stream=None):
    """Gradient of group_norm from its stats: (dx, dweight, dbias), the last two in float32 (None where there is no weight or bias), summed in a fixed order.  dx: where to
    (grad or x themselves, too)."""
    return _call(stream, _train.group_norm_backward, grad, x, groups, weight, bias, stats, _activation(activation), dx)


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, weight, bias, eps, activation):
        y, stats = _train.group_norm_forward(x, groups, weight, bias, eps, activation, None)
        ctx.save_for_backward(x, weight, bias, stats)
        ctx.how = groups, activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        x, weight, bias, stats = ctx.saved_tensors
        groups, activation = ctx.how
        dx, dw, db = _train.group_norm_backward(g.contiguous(), x, groups, weight, bias, stats, activation, None)
        return dx, None, dw.to(weight.dtype) if dw is not None else None, db.to(bias.dtype) if db is not None else None, None, None


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, activation=None, stream=None):
    """group_norm_forward's y, differentiable in x, weight and bias."""
    if torch.is_grad_enabled() and (getattr(x, "requires_grad", False) or getattr(weight, "requires_grad", False) or getattr(bias, "requires_grad", False)):
        return _call(stream, _GroupNorm.apply, x, groups, weight, bias, eps, _activation(activation))
    return group_norm_forward(x, groups, weight, bias, eps, activation, stream=stream)[0]


# ---- position bias ----

def _borders(e, c, f):
    """Where the coarse buckets 1 .. c - 1 of a side begin: the first distance x of x^c >= e^(c - j) f^j, which is found in 64-bit floats wherever they tell."""
    j = np.arange(1, c)
    at = e * (f / e) ** (j / c)                                # (to 2^-47 of itself)
    border = np.ceil(at).astype(np.int64)
    near = np.rint(at)
    for i in np.nonzero(np.abs(at - near) < 2.0 ** -40 * at)[0].tolist():
        x, g = int(near[i]), math.gcd(i + 1, c)
        p, q = (i + 1) // g, c // g
        # x = e (f / e)^(p / q) only with a q-th root of f / e that is a fraction of whole numbers below 2^25: q is 24 at most
        if q <= 24:
            border[i] = x if x ** q >= e ** (q - p) * f ** p else x + 1
        else:
            with localcontext() as precise:
                precise.prec = 60
                border[i] = x if q * Decimal(x).ln() >= (q - p) * Decimal(e).ln() + p * Decimal(f).ln() else x + 1
    return border


def position_buckets(exact, coarse=0, far=0, one_sided=False, device=0):
    """(buckets int32 [axes, 2 * reach + 1], their number) for position_bias.  On either side of an axis the distances below `exact` (0 among them) have a bucket each, those
    from `exact` to `far` share `coarse` buckets whose widths grow by a constant factor, and the last bucket takes all that is farther; one_sided: keys ahead of their query
    count as distance 0.  An axis' buckets follow each other from the farthest behind to the farthest ahead (one_sided: from distance 0 on), and those of several axes
    are combined with the last axis' together.  exact, coarse, far: numbers, or one for each axis: position_buckets((8, 8)) gives a bucket to every difference in a
    window of 8 x 8, position_buckets(8, 8, 128) is 31 buckets for one line of tokens.  Distances up to 2^24 and up to 2^24 buckets in all."""
    axes = max(len(v) if isinstance(v, (tuple, list)) else 1 for v in (exact, coarse, far))
    exact, coarse, far = ([int(n) for n in v] if isinstance(v, (tuple, list)) else [int(v)] * axes for v in (exact, coarse, far))
    if not len(exact) == len(coarse) == len(far) == axes or not 1 <= axes <= 4:
        raise ValueError("exact, coarse, far: one to four axes are wanted, a value for each")
    if any(e < 1 or c < 0 or (c and f <= e) for e, c, f in zip(exact, coarse, far)):
        raise ValueError("exact at least 1, coarse at least 0, and far above exact where there are coarse buckets, are wanted")
    reach = max(f if c else e - 1 for e, c, f in zip(exact, coarse, far))
    sides = [e + c if one_sided else 2 * (e + c) - 1 for e, c in zip(exact, coarse)]
    count = math.prod(sides)
    if reach > 2 ** 24 or count > 2 ** 24:                     # (what the library takes)
        raise ValueError("distances up to 2^24 and up to 2^24 buckets are wanted")
    rows, above = [], 1
    for e, c, f, n in reversed(list(zip(exact, coarse, far, sides))):
        borders = _borders(e, c, f) if c else np.empty(0, np.int64)
        x = np.arange(reach + 1)
        side = np.where(x < e, x, e + np.searchsorted(borders, x, side="right") if c else e - 1)
        last = e + c - 1
        row = np.concatenate([side[:0:-1], np.zeros(reach + 1, np.int64)] if one_sided else [last - side[:0:-1], last + side])
        rows.append((row * above).astype(np.int32))
        above *= n
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    return torch.from_numpy(np.stack(rows[::-1])).to(dev), count


class _PositionBias(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, positions, buckets, key_positions, segments, key_segments, dtype):
        ctx.save_for_backward(positions, buckets, key_positions, segments, key_segments)
        ctx.table = table.shape[0], table.dtype
        return _train.position_bias(table, positions, buckets, key_positions, segments, key_segments, dtype, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        positions, buckets, key_positions, segments, key_segments = ctx.saved_tensors
        count, dtype = ctx.table
        return (_train.position_bias_backward(_dense(g), positions, buckets, count, key_positions, segments, key_segments).to(dtype),) + (None,) * 6


def position_bias(table, positions, buckets, key_positions=None, segments=None, key_segments=None, dtype=None, out=None, stream=None):
    """A learned bias of attention for relative positions: [heads, queries, keys], or [batch, heads, queries, keys] where positions or segments are of several sequences.  table:
    [buckets, heads] of float32 or of the result's type (dtype, or the table's); positions (and key_positions, where keys are not the queries' tokens: a single new
    token against all before it): integers [axes, tokens] or [axes, batch, tokens], as patch_rows gives them; buckets: int32 [axes, 2 * reach + 1] (position_buckets).
    The pair's bucket is the sum over the axes of buckets[axis, reach + difference], the difference key - query held between -reach and reach; outside of the table it has no
    bias (0).  segments (and key_segments): int32 [tokens] or [batch, tokens], which of several packed sequences a token is of: pairs of different segments are -inf (a
    query of whose segment there is no key has a row of them), rows of queries whose segment is below 0 (padding) are 0.  out: where to, keys contiguous (rows may be padded); given, it keeps the call out of automatic differentiation."""
    kind = -1 if dtype is None else _TYPES.get(dtype, 3)
    if out is None and torch.is_grad_enabled() and getattr(table, "requires_grad", False):
        return _call(stream, _PositionBias.apply, table, positions, buckets, key_positions, segments, key_segments, kind)
    return _call(stream, _train.position_bias, table, positions, buckets, key_positions, segments, key_segments, kind, out)


def position_bias_backward(grad, positions, buckets, count, key_positions=None, segments=None, key_segments=None, stream=None):
    """Gradient of position_bias's table: float32 [count, heads], the sum of grad over the pairs of each bucket, in 64 bits, whose order is fixed as far as the GPU's own is
    (include/pcr.h).  What grad holds of pairs without a bias (of different segments, of padding) is not looked at."""
    return _call(stream, _train.position_bias_backward, grad, positions, buckets, count, key_positions, segments, key_segments)


# ---- dropout ----

def dropout_backward(grad, p, seed, call=0, dtype=None, out=None, stream=None):
    """Gradient of x of dropout(x, p, seed, call): grad, of the result's type, where x was kept, over the probability of that; of `dtype`, x's type (None: grad's)."""
    return _call(stream, _train.dropout, grad, p, seed, call, None, -1 if dtype is None else _TYPES.get(dtype, 3), out, False)[0]


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, call, residual):
        y, used = _train.dropout(x, p, seed, call, residual, -1, None, True)
        ctx.save_for_backward(used)
        ctx.how = p, call, _TYPES[x.dtype]
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        p, call, kind = ctx.how
        dx = _train.dropout(g.contiguous(), p, ctx.saved_tensors[0], call, None, kind, None, False)[0] if ctx.needs_input_grad[0] else None
        return dx, None, None, None, g if ctx.needs_input_grad[4] else None


def dropout(x, p, seed, call=0, residual=None, out=None, stream=None):
    """residual + x / (1 - p) where x is kept, residual (or 0) where it is dropped, each element with probability p; of residual's type, which is x's or float32.  No mask is
    stored: element e of x (in the order of its indexes) is dropped by word e of a counter-based generator (Philox4x32-10; include/pcr.h has the counters) for seed, an
    int64 CUDA tensor [2] of key and step, and call, 0 .. 65535, which tells the dropouts of one step apart.  The seed is read when the work runs (a captured graph may count
    its step up), and kept as it was read for the gradient.  x, residual: [..., dim], rows at one stride.  out: where to (x or residual themselves, too); given, it
    keeps the call out of automatic differentiation."""
    if out is None and torch.is_grad_enabled() and (getattr(x, "requires_grad", False) or getattr(residual, "requires_grad", False)):
        return _call(stream, _Dropout.apply, x, p, seed, call, residual)
    return _call(stream, _train.dropout, x, p, seed, call, residual, -1, out, False)[0]

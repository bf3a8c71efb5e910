"""The operators between a decoded record and a transformer that trains on it (include/pcr.h): patch rows and their positions, positions
of several axes turned into queries and keys (alone or behind a norm of every head), and distillation from a teacher's top logits.

The work is done by the library's HIP kernels, enqueued on the current stream (or `stream`, a hipStream_t as an integer); arguments are checked and handed on
by the native module _train (csrc/pcr_bind.cpp).  A tensor on another stream than the one it was made on needs the caller's
record_stream, as with any operator.  Wrong types, shapes or devices raise ValueError before anything is enqueued, what the library
refuses raises PcrError.  rotate_axes, norm_rotate and distill_loss take part in automatic differentiation; a gradient is made on the stream of its forward pass.
There are no derivatives of forward mode (ValueError), and no traces (RuntimeError)."""
import os

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

"""The operators between a decoded record and a transformer that trains on it (include/pcr.h): patch rows and their positions, positions
of several axes turned into queries and keys (alone or behind a norm of every head), and distillation from a teacher's top logits.

As in binding.py the functions here check and marshal arguments; the work is done by the library's HIP kernels, enqueued on the current
stream (or `stream`, a hipStream_t as an integer).  A tensor on another stream than the one it was made on needs the caller's
record_stream, as with any operator.  Wrong types, shapes or devices raise ValueError before anything is enqueued, what the library
refuses raises PcrError.  rotate_axes, norm_rotate and distill_loss take part in automatic differentiation."""
import ctypes
import math

import numpy as np
import torch

from .binding import _check, lib

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_i64, _vp = ctypes.c_int64, ctypes.c_void_p


class _Heads(ctypes.Structure):
    _fields_ = [("in_", _vp), ("in_batch", _i64), ("in_token", _i64), ("in_head", _i64),
                ("out", _vp), ("out_batch", _i64), ("out_token", _i64), ("out_head", _i64),
                ("grad", _vp), ("grad_batch", _i64), ("grad_token", _i64), ("grad_head", _i64),
                ("weight", _vp), ("weight_grad", _vp), ("heads", _i64)]


class _Rotation(ctypes.Structure):
    _fields_ = [("position", _vp), ("axis_stride", _i64), ("batch_stride", _i64), ("token_stride", _i64), ("frequency", _vp), ("axis", _vp),
                ("batch", _i64), ("tokens", _i64), ("wide", ctypes.c_int32), ("axes", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("pairs", ctypes.c_int32), ("adjacent", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _Distill(ctypes.Structure):
    _fields_ = [("logits", _vp), ("row_stride", _i64), ("top_index", _vp), ("top_logits", _vp), ("labels", _vp), ("rows", _i64), ("classes", _i64),
                ("top", ctypes.c_int32), ("dtype", ctypes.c_int32), ("top_dtype", ctypes.c_int32), ("index_wide", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("distill_part", ctypes.c_float), ("label_part", ctypes.c_float), ("reserved", ctypes.c_float)]


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _on(t, device, what):
    _need(t.is_cuda and t.device == device, "%s: a tensor on %s is wanted" % (what, device))


def _stream(device, stream):
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


# ---- patch rows ----

def patch_layout(shapes, channels, patch, merge=1, offsets=None, device=0):
    """What patch_rows needs to know of pictures of the given (height, width), one behind the other as decode_batch writes them (offsets: where
    each begins, and the end): (shapes int32 [n, 2], offsets int64 [n + 1], first_rows int64 [n + 1]) as CUDA tensors, and the number of rows."""
    hw = np.asarray(shapes, np.int64).reshape(-1, 2)
    cell = patch * merge
    rows = np.where((hw > 0).all(1), (-(-hw // cell) * merge).prod(1), 0)
    if offsets is None:
        offsets = np.concatenate([[0], np.cumsum(hw.prod(1) * channels)])
    first = np.concatenate([[0], np.cumsum(rows)])
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    return (torch.from_numpy(hw.astype(np.int32)).to(dev), torch.from_numpy(np.asarray(offsets).astype(np.int64)).to(dev),
            torch.from_numpy(first.astype(np.int64)).to(dev), int(first[-1]))


def patch_rows(pixels, shapes, offsets, first_rows, rows, patch, mean, inv_std, merge=1, frames=1, dtype=torch.bfloat16, out=None, positions=None,
               stream=None):
    """Normalised patch rows of ragged uint8 pictures (decode_batch's pixels; shapes, offsets and first_rows from patch_layout), and their
    positions: (dtype [rows, channels * patch * patch], int32 [3, rows]: frame, row, column).  channels = len(mean), 1 or 3; see
    pcr_patch_rows for the order of the rows and for merge and frames."""
    dev = pixels.device
    C, n = len(mean), shapes.shape[0]
    _need(pixels.is_cuda and pixels.dtype == torch.uint8 and pixels.is_contiguous(), "pixels: a contiguous uint8 CUDA tensor is wanted")
    for t, kind, shape, what in ((shapes, torch.int32, (n, 2), "shapes"), (offsets, torch.int64, (n + 1,), "offsets"), (first_rows, torch.int64, (n + 1,), "first_rows")):
        _on(t, dev, what)
        _need(t.dtype == kind and tuple(t.shape) == shape and t.is_contiguous(), "%s: contiguous %s %s is wanted" % (what, kind, list(shape)))
    _need(C in (1, 3) and len(inv_std) == C, "mean and inv_std: one or three values each")
    _need(rows >= 0 and patch >= 1 and merge >= 1 and frames >= 1, "rows, patch, merge, frames: out of range")
    if out is None:
        _need(dtype in _TYPES, "dtype: float32, float16 or bfloat16 is wanted")
        out = torch.empty((rows, C * patch * patch), dtype=dtype, device=dev)
    if positions is None:
        positions = torch.empty((3, rows), dtype=torch.int32, device=dev)
    _on(out, dev, "out")
    _on(positions, dev, "positions")
    _need(out.dtype in _TYPES and out.is_contiguous() and out.numel() == rows * C * patch * patch, "out: contiguous [rows, channels * patch * patch] is wanted")
    _need(positions.dtype == torch.int32 and positions.is_contiguous() and tuple(positions.shape) == (3, rows), "positions: contiguous int32 [3, rows] is wanted")
    m = (ctypes.c_float * 3)(*mean)
    s = (ctypes.c_float * 3)(*inv_std)
    _check(lib().pcr_patch_rows(dev.index, pixels.data_ptr(), pixels.numel(), shapes.data_ptr(), offsets.data_ptr(), first_rows.data_ptr(), n, rows, patch, merge, frames, C,
                                m, s, _TYPES[out.dtype], out.data_ptr(), positions.data_ptr(), _stream(dev, stream)), "pcr_patch_rows")
    return out, positions


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


def _rotation(x, positions, frequency, axis, adjacent):
    """The structure for heads like x, [tokens, heads, dim] or [batch, tokens, heads, dim]."""
    dev = x.device
    batch, tokens = (1, x.shape[0]) if x.dim() == 3 else x.shape[:2]
    _on(positions, dev, "positions")
    _on(frequency, dev, "frequency")
    _on(axis, dev, "axis")
    kind = positions.dtype
    _need(kind == torch.int32 or kind == torch.int64, "positions: int32 or int64 is wanted")
    pairs = frequency.shape[0] if frequency.dim() == 1 else -1
    _need(frequency.dtype == torch.float32 and axis.dtype == torch.int32 and frequency.is_contiguous() and axis.is_contiguous()
          and pairs >= 0 and axis.dim() == 1 and axis.shape[0] == pairs, "frequency and axis: contiguous float32 [pairs] and int32 [pairs] are wanted")
    _need(2 * pairs <= x.shape[-1], "frequency: more pairs than half of a head")
    shape = positions.shape
    if len(shape) == 2:                                    # the same for every sequence
        _need(shape[1] == tokens, "positions: [axes, tokens] is wanted")
        sa, sb, st = positions.stride(0), 0, positions.stride(1)
    else:
        _need(len(shape) == 3 and shape[1] == batch and shape[2] == tokens, "positions: [axes, tokens] or [axes, batch, tokens] is wanted")
        sa, sb, st = positions.stride()
    _need(1 <= shape[0] <= 4, "positions: one to four axes are wanted")
    return _Rotation(positions.data_ptr(), sa, sb, st, frequency.data_ptr(), axis.data_ptr(), batch, tokens, kind == torch.int64, shape[0], x.shape[-1],
                     pairs, bool(adjacent), 0)


def _places(t):
    """(pointer, batch, token, head strides)"""
    st = t.stride()
    return (t.data_ptr(), 0, st[0], st[1]) if t.dim() == 3 else (t.data_ptr(), st[0], st[1], st[2])


_NOWHERE = (None, 0, 0, 0)


def _like(t, x, what):
    _on(t, x.device, what)
    _need(t.dtype == x.dtype and t.shape == x.shape and (t.stride(-1) == 1 or t.shape[-1] == 1), "%s: %s %s is wanted, with each head's elements contiguous" % (what, x.dtype, list(x.shape)))


def _into(t, x, what):
    _like(t, x, what)
    _need(all(st or n < 2 for st, n in zip(t.stride(), t.shape)), "%s: every element needs a place of its own" % what)


def _side(x, out, grad=None, weight=None, weight_grad=None):
    if x is None:
        return _Heads()
    return _Heads(*_places(x), *_places(out), *(_places(grad) if grad is not None else _NOWHERE), weight.data_ptr() if weight is not None else None,
                  weight_grad.data_ptr() if weight_grad is not None else None, x.shape[-2])


def _check_heads(q, k):
    _need(q.is_cuda and q.dtype in _TYPES and q.dim() in (3, 4), "q: float32, float16 or bfloat16 [(batch,) tokens, heads, dim] on the GPU is wanted")
    _like(q, q, "q")
    if k is not None:
        _need(k.dim() == q.dim() and k.shape[:-2] == q.shape[:-2] and k.shape[-1] == q.shape[-1], "k: the batch, tokens and dim of q are wanted")
        _like(k, k, "k")
        _need(k.dtype == q.dtype and k.device == q.device, "k: type and device of q are wanted")


def _outs(q, k, q_out, k_out):
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _into(q_out, q, "q_out")
    if k is not None:
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        else:
            _into(k_out, k, "k_out")
    return q_out, k_out


def _weight(w, x, what):
    if w is not None:
        _on(w, x.device, what)
        _need(w.dim() == 1 and w.shape[0] == x.shape[-1] and w.is_contiguous() and w.dtype in (torch.float32, x.dtype), "%s: contiguous [dim] of float32 or the heads' type is wanted" % what)


def _rotate(q, k, positions, frequency, axis, adjacent, inverse, q_out, k_out, stream):
    _check_heads(q, k)
    q_out, k_out = _outs(q, k, q_out, k_out)
    R = _rotation(q, positions, frequency, axis, adjacent)
    a, b = _side(q, q_out), _side(k, k_out)
    _check(lib().pcr_rotate_axes(q.device.index, ctypes.byref(a), ctypes.byref(b), ctypes.byref(R), int(inverse), _TYPES[q.dtype], _stream(q.device, stream)),
           "pcr_rotate_axes")
    return q_out, k_out


class _RotateAxes(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, frequency, axis, adjacent, inverse):
        ctx.save_for_backward(positions, frequency, axis)
        ctx.how = adjacent, inverse, q.shape, k.shape if k is not None else None
        return _rotate(q, k, positions, frequency, axis, adjacent, inverse, None, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        adjacent, inverse, _, kshape = ctx.how
        gq, gk = _dense(gq), _dense(gk) if kshape is not None else None
        dq, dk = _rotate(gq, gk, *ctx.saved_tensors, adjacent, not inverse, None, None, None)
        return dq, dk, None, None, None, None, None


def _dense(g):
    """A gradient as a broadcast view may come with strides of 0, which is read as it is; only a head's elements have to follow each other."""
    return g if g.stride(-1) == 1 or g.shape[-1] == 1 else g.contiguous()


def rotate_axes(q, k, positions, frequency, axis, adjacent=False, inverse=False, q_out=None, k_out=None, stream=None):
    """Turns the pairs of queries and keys by positions of up to four axes: pair j of a token's heads by positions[axis[j]] * frequency[j] radians.
    q, k: [tokens, heads, dim] or [batch, tokens, heads, dim] (k may be None) with any strides of batch, tokens and heads; positions: integers [axes,
    tokens] or [axes, batch, tokens].  A pair is (j, j + pairs), or (2 j, 2 j + 1) if `adjacent`; what is behind the pairs is not turned.  inverse:
    by minus the angle, which is the gradient.  q_out, k_out: where to (the inputs themselves, too); given, they keep the call out of automatic
    differentiation.  Returns (q, k) turned."""
    if q_out is None and k_out is None and stream is None and torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad)):
        return _RotateAxes.apply(q, k, positions, frequency, axis, adjacent, inverse)
    return _rotate(q, k, positions, frequency, axis, adjacent, inverse, q_out, k_out, stream)


def _norm(q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, q_out, k_out, stream):
    _check_heads(q, k)
    _need(eps >= 0, "eps: not below 0")
    wdtype = _weights(q, k, q_weight, k_weight)
    q_out, k_out = _outs(q, k, q_out, k_out)
    R = _rotation(q, positions, frequency, axis, adjacent)
    a, b = _side(q, q_out, None, q_weight), _side(k, k_out, None, k_weight)
    _check(lib().pcr_norm_rotate(q.device.index, ctypes.byref(a), ctypes.byref(b), ctypes.byref(R), eps, _TYPES[q.dtype], _TYPES[wdtype],
                                 _stream(q.device, stream)), "pcr_norm_rotate")
    return q_out, k_out


def _weights(q, k, q_weight, k_weight):
    """The weights' common type."""
    _weight(q_weight, q, "q_weight")
    _weight(k_weight, q, "k_weight")
    _need(k is not None or k_weight is None, "k_weight without k")
    kinds = {w.dtype for w in (q_weight, k_weight) if w is not None}
    _need(len(kinds) < 2, "q_weight and k_weight: one type is wanted")
    return kinds.pop() if kinds else q.dtype


def norm_rotate_backward(gq, gk, q, k, q_weight, k_weight, positions, frequency, axis, eps=1e-6, adjacent=False, dq=None, dk=None, stream=None):
    """Gradient of norm_rotate: (dq, dk, dq_weight, dk_weight), the weights' in float32 (None where there is no weight), summed in a fixed order.  gq and gk: the
    gradients of its results; dq and dk: where to (gq and gk, or q and k, themselves, too)."""
    _check_heads(q, k)
    _need(eps >= 0, "eps: not below 0")
    wdtype = _weights(q, k, q_weight, k_weight)
    _need((gk is None) == (k is None), "gk: one for k")
    _like(gq, q, "gq")
    if k is not None:
        _like(gk, k, "gk")
    dq, dk = _outs(q, k, dq, dk)
    R = _rotation(q, positions, frequency, axis, adjacent)
    dev, dim = q.device, q.shape[-1]
    sums = torch.empty((2, dim), dtype=torch.float32, device=dev)
    dqw = sums[0] if q_weight is not None else None
    dkw = sums[1] if k_weight is not None else None
    need = ctypes.c_size_t(0)
    _check(lib().pcr_norm_rotate_workspace(R.batch * R.tokens, dim, ctypes.byref(need)), "pcr_norm_rotate_workspace")
    work = torch.empty(need.value, dtype=torch.uint8, device=dev)
    a, b = _side(q, dq, gq, q_weight, dqw), _side(k, dk, gk, k_weight, dkw)
    _check(lib().pcr_norm_rotate_backward(dev.index, ctypes.byref(a), ctypes.byref(b), ctypes.byref(R), eps, _TYPES[q.dtype], _TYPES[wdtype],
                                          work.data_ptr(), need.value, _stream(dev, stream)), "pcr_norm_rotate_backward")
    return dq, dk, dqw, dkw


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, frequency, axis)
        ctx.how = eps, adjacent
        return _norm(q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, None, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        q, k, q_weight, k_weight, positions, frequency, axis = ctx.saved_tensors
        dq, dk, dqw, dkw = norm_rotate_backward(_dense(gq), _dense(gk) if k is not None else None, q, k, q_weight, k_weight, positions, frequency, axis, *ctx.how)
        return (dq, dk, dqw.to(q_weight.dtype) if dqw is not None else None, dkw.to(k_weight.dtype) if dkw is not None else None) + (None,) * 5


def norm_rotate(q, k, q_weight, k_weight, positions, frequency, axis, eps=1e-6, adjacent=False, q_out=None, k_out=None, stream=None):
    """rotate_axes of x * weight / sqrt(mean x^2 + eps), the mean over each head of queries and keys, in one pass and with one rounding.  Weights: [dim]
    of float32 or of the heads' type, or None.  Returns (q, k)."""
    if q_out is None and k_out is None and stream is None and torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, q_weight, k_weight)):
        return _NormRotate.apply(q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent)
    return _norm(q, k, q_weight, k_weight, positions, frequency, axis, eps, adjacent, q_out, k_out, stream)


# ---- distillation ----

def _distill(logits, top_index, top_logits, labels, temperature, distill_part, label_part):
    dev = logits.device
    _need(logits.is_cuda and logits.dtype in _TYPES and logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1), "logits: float32, float16 or bfloat16 [rows, classes] on the GPU, a row contiguous, is wanted")
    rows, classes = logits.shape
    _on(top_index, dev, "top_index")
    _on(top_logits, dev, "top_logits")
    _need(top_index.dim() == 2 and top_index.shape[0] == rows and top_index.dtype in (torch.int32, torch.int64) and top_index.is_contiguous(), "top_index: contiguous int32 or int64 [rows, top] is wanted")
    _need(top_logits.shape == top_index.shape and top_logits.dtype in _TYPES and top_logits.is_contiguous(), "top_logits: contiguous, of top_index's shape, is wanted")
    if labels is not None:
        _on(labels, dev, "labels")
        _need(labels.dtype == torch.int64 and tuple(labels.shape) == (rows,) and labels.is_contiguous(), "labels: contiguous int64 [rows] is wanted")
    _need(temperature > 0 and math.isfinite(temperature), "temperature: above 0")
    return _Distill(logits.data_ptr(), logits.stride(0), top_index.data_ptr(), top_logits.data_ptr(), labels.data_ptr() if labels is not None else None,
                    rows, classes, top_index.shape[1], _TYPES[logits.dtype], _TYPES[top_logits.dtype], top_index.dtype == torch.int64,
                    temperature, distill_part, label_part, 0.0)


def _distill_work(d, dev):
    need = ctypes.c_size_t(0)
    _check(lib().pcr_distill_workspace(d.rows, d.classes, ctypes.byref(need)), "pcr_distill_workspace")
    return (torch.empty(need.value, dtype=torch.uint8, device=dev), need.value) if need.value else (None, 0)


def _rows_of(t, logits, what):
    _on(t, logits.device, what)
    _need(t.dtype == torch.float32 and tuple(t.shape) == (logits.shape[0],) and t.is_contiguous(), "%s: contiguous float32 [rows] is wanted" % what)


def _gradient_out(out, logits):
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _on(out, logits.device, "out")
    _need(out.dtype == logits.dtype and out.shape == logits.shape and (out.stride(1) == 1 or out.shape[1] == 1), "out: type and shape of logits, a row contiguous, is wanted")
    return out


def distill_forward(logits, top_index, top_logits, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, stream=None):
    """(loss float32 [rows], sums float32 [rows, 2]): of every row distill_part * temperature^2 * the divergence of softmax(logits / temperature) from the
    softmax of the teacher's kept logits (top_logits / temperature at classes top_index; a class outside 0 .. classes - 1 does not count), and label_part
    * the cross entropy with labels (int64; one outside the classes does not count).  sums is what distill_backward takes."""
    d = _distill(logits, top_index, top_logits, labels, temperature, distill_part, label_part)
    dev = logits.device
    loss = torch.empty(d.rows, dtype=torch.float32, device=dev)
    sums = torch.empty((d.rows, 2), dtype=torch.float32, device=dev)
    work, nbytes = _distill_work(d, dev)
    _check(lib().pcr_distill_forward(dev.index, ctypes.byref(d), loss.data_ptr(), sums.data_ptr(), work.data_ptr() if nbytes else None, nbytes,
                                     _stream(dev, stream)), "pcr_distill_forward")
    return loss, sums


def distill_backward(row_grad, logits, top_index, top_logits, sums, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, out=None, stream=None):
    """The gradient of the logits for row_grad, the gradient of every row's loss (float32 [rows]), from distill_forward's sums.  out: where to (the logits
    themselves, too)."""
    d = _distill(logits, top_index, top_logits, labels, temperature, distill_part, label_part)
    _rows_of(row_grad, logits, "row_grad")
    _on(sums, logits.device, "sums")
    _need(sums.dtype == torch.float32 and tuple(sums.shape) == (d.rows, 2) and sums.is_contiguous(), "sums: contiguous float32 [rows, 2] is wanted")
    out = _gradient_out(out, logits)
    dev = logits.device
    _check(lib().pcr_distill_backward(dev.index, ctypes.byref(d), sums.data_ptr(), row_grad.data_ptr(), out.data_ptr(), out.stride(0), _stream(dev, stream)),
           "pcr_distill_backward")
    return out


def distill_step(logits, top_index, top_logits, row_weight, labels=None, temperature=1.0, distill_part=1.0, label_part=0.0, out=None, stream=None):
    """(loss, gradient) in one pass: loss[n] = row_weight[n] * distill_forward's loss, and the gradient of their sum.  A row of weight 0 is left out whatever
    it holds.  out: where the gradient goes (the logits themselves, too)."""
    d = _distill(logits, top_index, top_logits, labels, temperature, distill_part, label_part)
    _rows_of(row_weight, logits, "row_weight")
    out = _gradient_out(out, logits)
    dev = logits.device
    loss = torch.empty(d.rows, dtype=torch.float32, device=dev)
    work, nbytes = _distill_work(d, dev)
    _check(lib().pcr_distill_step(dev.index, ctypes.byref(d), row_weight.data_ptr(), loss.data_ptr(), out.data_ptr(), out.stride(0),
                                  work.data_ptr() if nbytes else None, nbytes, _stream(dev, stream)), "pcr_distill_step")
    return loss, out


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

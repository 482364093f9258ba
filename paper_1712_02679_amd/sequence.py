"""ctypes binding of include/adacomp_sequence.h: embedding, gated linear recurrence and distillation, forward and backward.

Argument marshalling and checks only, in the manner of layers.py: the caller makes all tensors, results included, on the current device, and
the calls run on torch's current stream.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, lib
from .layers import (_DTYPES, _Dropout, _current_stream, _device_of, _drop, _f32, _i64, _in_32_bits, _per_sequence, _refuse, _room, _rows, _sz, _u32,
                     _u64, _unlike, _vector, _vp)

SEQUENCE_EXPORTS = [
    "adacomp_embed_forward", "adacomp_embed_workspace_bytes", "adacomp_embed_backward", "adacomp_recurrence_workspace_bytes",
    "adacomp_recurrence_forward", "adacomp_recurrence_backward", "adacomp_distill_forward", "adacomp_distill_backward",
]

RECURRENCE_KEEP = 64
TEACHER_TOP_MAX = 256

_INDEX_BYTES = {torch.int32: 4, torch.int64: 8}


class _Embed(ctypes.Structure):
    _fields_ = [("rows", _u64), ("stride", _u64), ("vocab", _u32), ("cols", _u32), ("dtype", _u32), ("index_bytes", _u32), ("tokens", _vp), ("scale", _f32),
                ("reserved", _u32)]


class _Steps(ctypes.Structure):
    _fields_ = [("data", _vp), ("batch_stride", _i64), ("row_stride", _i64)]


class _Recurrence(ctypes.Structure):
    _fields_ = [("batch", _u32), ("length", _u32), ("channels", _u32), ("dtype", _u32), ("bias", _vp), ("lengths", _vp), ("resets", _vp), ("resets_stride", _i64)]


class _Distill(ctypes.Structure):
    _fields_ = [("rows", _u64), ("vocab", _u32), ("dtype", _u32), ("logits_stride", _u64), ("dlogits_stride", _u64), ("teacher_tokens", _vp),
                ("teacher_logits", _vp), ("targets", _vp), ("tokens_stride", _u64), ("teacher_stride", _u64), ("top", _u32), ("teacher_dtype", _u32),
                ("tokens_bytes", _u32), ("targets_bytes", _u32), ("temperature", _f32), ("soft", _f32), ("hard", _f32), ("scale", _f32)]


_bound = None   # the library, once it has the argument types below


def _lib():
    """The library with the argument types of these calls."""
    global _bound
    if _bound is None:
        L = lib()
        P, i32 = ctypes.POINTER, ctypes.c_int
        L.adacomp_embed_forward.argtypes = [P(_Embed), _vp, _vp, P(_Dropout), _vp]
        L.adacomp_embed_workspace_bytes.argtypes, L.adacomp_embed_workspace_bytes.restype = [_u64, _u32, _u32], _sz
        L.adacomp_embed_backward.argtypes = [P(_Embed), _vp, _vp, P(_Dropout), i32, _vp, _sz, _vp]
        L.adacomp_recurrence_workspace_bytes.argtypes, L.adacomp_recurrence_workspace_bytes.restype = [_u32] * 3, _sz
        L.adacomp_recurrence_forward.argtypes = [P(_Recurrence), P(_Steps), P(_Steps), P(_Steps), _vp, P(_Steps), _vp, _vp, _vp, _sz, _vp]
        L.adacomp_recurrence_backward.argtypes = [P(_Recurrence), P(_Steps), P(_Steps), P(_Steps), P(_Steps), _vp, _vp, P(_Steps), P(_Steps), P(_Steps), _vp, _vp, i32,
                                                  _vp, _sz, _vp]
        L.adacomp_distill_forward.argtypes = [P(_Distill), _vp, _vp, _vp, _vp, _vp, _vp]
        L.adacomp_distill_backward.argtypes = [P(_Distill), _vp, _vp, _vp, _vp, _vp]
        _bound = L
    return _bound


def _type_of(x, what):
    number = _DTYPES.get(x.dtype)
    if number is None:
        _refuse(f"{what}: {x.dtype} is not one of float32, bfloat16, float16")
    return number


# ---- embedding ------------------------------------------------------------------------------------------------------

def _embed(tokens, rows, table, scale, what):
    """(the operator, address of the rows, of the table, device)"""
    number, dev = _type_of(rows, what), _device_of(rows)
    shape = rows.shape
    if table.dim() != 2 or table.dtype is not torch.float32 or not table.is_contiguous() or table.get_device() != dev:
        _refuse(f"table: a contiguous float32 tensor [vocab, columns] on the device of {what} is wanted")
    vocab, cols = table.shape
    index = _INDEX_BYTES.get(tokens.dtype)
    if index is None or not tokens.is_contiguous() or tokens.get_device() != dev:
        _refuse(f"tokens: a contiguous tensor of int32 or int64 on the device of {what} is wanted")
    if shape != (*tokens.shape, cols):
        _unlike(rows, (*tokens.shape, cols), rows.dtype, what)
    if (vocab | cols) >> 32:
        _refuse(f"table: {tuple(table.shape)}: not all are numbers of 32 bits")
    address, stride = _rows(rows, shape, rows.dtype, dev, what)
    return _Embed(tokens.numel(), stride, vocab, cols, number, index, tokens.data_ptr(), scale, 0), address, table.data_ptr(), dev


def adacomp_embed_forward(tokens, table, y, scale=1.0, dropout=None):
    """y = D(scale * table[tokens]), zeros where a number is no token of the table.  table [vocab, columns] float32 may be a part of the flat
    weights; y has the tokens' shape and the columns behind it."""
    L = _bound or _lib()
    op, py, pt, dev = _embed(tokens, y, table, scale, "y")
    rc = L.adacomp_embed_forward(op, pt, py, _drop(dropout, dev), _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_embed_workspace_bytes(rows, vocab, cols) -> int:
    sizes = [int(n) for n in (rows, vocab, cols)]
    return int(_lib().adacomp_embed_workspace_bytes(*sizes)) if all(0 <= n < 2 ** 32 for n in sizes) else 0


def adacomp_embed_backward(tokens, dy, dtable, workspace, scale=1.0, dropout=None, accumulate=False):
    """dtable (a part of the flat gradient): the sum of scale * D(dy) over the places of each token, all of it overwritten, or with accumulate
    added to.  Made for mini-batches: beyond some 100000 places the time grows with places times vocabulary (see adacomp_sequence.h)."""
    L = _bound or _lib()
    op, pdy, pt, dev = _embed(tokens, dy, dtable, scale, "dy")
    pw, nw = _room(workspace, dev)
    rc = L.adacomp_embed_backward(op, pdy, pt, _drop(dropout, dev), 1 if accumulate else 0, pw, nw, _current_stream(dev))
    if rc:
        _check(rc)


# ---- gated linear recurrence ----------------------------------------------------------------------------------------

def _steps(t, shape, dtype, device, what):
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _unlike(t, shape, dtype, what)
    b, n, c = t.stride()
    if c != 1 and shape[2] > 1:
        _refuse(f"{what}: the last dimension is not contiguous")
    return _Steps(t.data_ptr(), b, n)


def _recurrence(x, bias, lengths, resets):
    """(the operator, shape, type and device of its tensors)"""
    shape, number = x.shape, _type_of(x, "x")
    if len(shape) != 3:
        _refuse("x: [batch, length, channels] is wanted")
    dev = _device_of(x)
    b, n, c = shape
    if (b | n | c) >> 32:
        _refuse(f"sizes {tuple(shape)}: not all are numbers of 32 bits")
    address = stride = None
    if resets is not None:
        if resets.dtype not in (torch.uint8, torch.bool) or resets.shape != (b, n) or resets.get_device() != dev or resets.stride(1) != 1 and n > 1:
            _refuse(f"resets: a uint8 or bool tensor {(b, n)} on the device of x, with a contiguous last dimension, is wanted")
        address, stride = resets.data_ptr(), resets.stride(0)
    op = _Recurrence(b, n, c, number, _vector(bias, c, dev, "bias"), _per_sequence(lengths, b, dev, "lengths"), address, stride or 0)
    return op, shape, x.dtype, dev


def adacomp_recurrence_kept(length) -> int:
    """States that the forward pass keeps of a sequence."""
    return (int(length) + RECURRENCE_KEEP - 1) // RECURRENCE_KEEP


def adacomp_recurrence_workspace_bytes(batch, length, channels) -> int:
    sizes = [int(n) for n in (batch, length, channels)]
    return int(_lib().adacomp_recurrence_workspace_bytes(*sizes)) if all(0 <= n < 2 ** 32 for n in sizes) else 0


def adacomp_recurrence_forward(x, forget, y, workspace, out=None, bias=None, first=None, last=None, states=None, lengths=None, resets=None):
    """h = m h + (1 - a) x along each sequence of x [batch, length, channels] with a = sigmoid(forget + bias), y = sigmoid(out) h (see
    adacomp_sequence.h).  first and last, [batch, channels] float32, are the states before and behind the sequences and may be one tensor;
    states [batch, adacomp_recurrence_kept(length), channels] float32 is for the backward pass."""
    L = _bound or _lib()
    op, shape, dtype, dev = _recurrence(x, bias, lengths, resets)
    b, n, c = shape
    pw, nw = _room(workspace, dev)
    rc = L.adacomp_recurrence_forward(op, _steps(x, shape, dtype, dev, "x"), _steps(forget, shape, dtype, dev, "forget"), _steps(out, shape, dtype, dev, "out"),
                                      _vector(first, b * c, dev, "first"), _steps(y, shape, dtype, dev, "y"), _vector(last, b * c, dev, "last"),
                                      _vector(states, b * adacomp_recurrence_kept(n) * c, dev, "states"), pw, nw, _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_recurrence_backward(dy, x, forget, states, dx, dforget, workspace, out=None, dout=None, bias=None, dbias=None, dlast=None, dfirst=None,
                                lengths=None, resets=None, accumulate=False):
    """dx, dforget, dout (with out), dbias (a part of the flat gradient: overwritten, or with accumulate added to) and dfirst from dy and dlast,
    with the other arguments and the states of the forward pass."""
    L = _bound or _lib()
    op, shape, dtype, dev = _recurrence(x, bias, lengths, resets)
    b, n, c = shape
    pw, nw = _room(workspace, dev)
    view = lambda t, what: _steps(t, shape, dtype, dev, what)
    rc = L.adacomp_recurrence_backward(op, view(dy, "dy"), view(x, "x"), view(forget, "forget"), view(out, "out"),
                                       _vector(states, b * adacomp_recurrence_kept(n) * c, dev, "states"), _vector(dlast, b * c, dev, "dlast"), view(dx, "dx"),
                                       view(dforget, "dforget"), view(dout, "dout"), _vector(dbias, c, dev, "dbias"), _vector(dfirst, b * c, dev, "dfirst"),
                                       1 if accumulate else 0, pw, nw, _current_stream(dev))
    if rc:
        _check(rc)


# ---- distillation ---------------------------------------------------------------------------------------------------

def _top_rows(t, rows, top, device, what):
    """Row stride of a [rows, top] tensor, whose leading dimensions may be several."""
    if t.get_device() != device or t.dim() < 1 or t.shape[-1] != top or t.numel() != rows * top:
        _unlike(t, (rows, top), t.dtype, what)
    return _rows(t, t.shape, t.dtype, device, what)


def _distill(logits, dlogits, teacher_tokens, teacher_logits, targets, temperature, soft, hard, scale):
    """(the operator, addresses of logits and dlogits, rows, device)"""
    number, dev, shape = _type_of(logits, "logits"), _device_of(logits), logits.shape
    if not shape:
        _refuse("logits: no dimension")
    vocab = shape[-1]
    rows = logits.numel() // vocab if vocab else 0
    if vocab >> 32:
        _in_32_bits(vocab, "vocabulary")
    pz, sz = _rows(logits, shape, logits.dtype, dev, "logits")
    pd, sd = _rows(dlogits, shape, logits.dtype, dev, "dlogits")
    op = _Distill(rows, vocab, number, sz, sd, temperature=temperature, soft=soft, hard=hard, scale=scale)
    if (teacher_tokens is None) != (teacher_logits is None):
        _refuse("teacher_tokens and teacher_logits go together")
    if teacher_tokens is not None:
        if not teacher_tokens.shape:
            _refuse("teacher_tokens: no dimension")
        index, top = _INDEX_BYTES.get(teacher_tokens.dtype), teacher_tokens.shape[-1]
        if index is None:
            _refuse(f"teacher_tokens: {teacher_tokens.dtype} is not one of int32, int64")
        if top >> 32:
            _in_32_bits(top, "top tokens")
        op.teacher_tokens, op.tokens_stride = _top_rows(teacher_tokens, rows, top, dev, "teacher_tokens")
        op.teacher_dtype = _type_of(teacher_logits, "teacher_logits")
        op.teacher_logits, op.teacher_stride = _top_rows(teacher_logits, rows, top, dev, "teacher_logits")
        op.top, op.tokens_bytes = top, index
    if targets is not None:
        index = _INDEX_BYTES.get(targets.dtype)
        if index is None or targets.numel() != rows or not targets.is_contiguous() or targets.get_device() != dev:
            _refuse(f"targets: a contiguous tensor of {rows} int32 or int64 numbers on the device of the logits is wanted")
        op.targets, op.targets_bytes = targets.data_ptr(), index
    return op, pz, pd, rows, dev


def adacomp_distill_forward(logits, loss, lse=None, teacher_tokens=None, teacher_logits=None, targets=None, temperature=1.0, soft=1.0, hard=1.0,
                            dlogits=None, dloss=None, scale=1.0):
    """The loss of every row of logits [..., vocab]: soft * temperature^2 * KL(teacher || student) over the teacher's top tokens, [..., top], plus
    hard * cross entropy with the targets (see adacomp_sequence.h).  loss has a float32 for every row, lse two, for the backward pass.  With
    dlogits the gradient of scale * sum(dloss * loss) is computed at the same time; dloss is ones where it is None."""
    L = _bound or _lib()
    op, pz, pd, rows, dev = _distill(logits, dlogits, teacher_tokens, teacher_logits, targets, temperature, soft, hard, scale)
    rc = L.adacomp_distill_forward(op, pz, _vector(loss, rows, dev, "loss"), _vector(lse, 2 * rows, dev, "lse"), _vector(dloss, rows, dev, "dloss"), pd,
                                   _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_distill_backward(logits, lse, dlogits, dloss=None, teacher_tokens=None, teacher_logits=None, targets=None, temperature=1.0, soft=1.0, hard=1.0,
                             scale=1.0):
    """dlogits, which may be the logits' buffer, from the lse of the forward pass and its other arguments."""
    L = _bound or _lib()
    op, pz, pd, rows, dev = _distill(logits, dlogits, teacher_tokens, teacher_logits, targets, temperature, soft, hard, scale)
    rc = L.adacomp_distill_backward(op, pz, _vector(lse, 2 * rows, dev, "lse"), _vector(dloss, rows, dev, "dloss"), pd, _current_stream(dev))
    if rc:
        _check(rc)

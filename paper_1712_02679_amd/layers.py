"""ctypes binding of include/adacomp_layers.h: dropout, layer norm and the biased softmax, forward and backward.

Argument marshalling and checks only; everything is computed by the HIP kernels behind the calls.  Tensors are float32,
bfloat16 or float16 on the current device (parameters, their gradients and statistics float32), the caller makes all
of them, results included, and the calls run on torch's current stream.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from .binding import EINVAL, AdacompError, _check, lib

LAYER_EXPORTS = [
    "adacomp_dropout", "adacomp_norm_forward", "adacomp_norm_workspace_bytes", "adacomp_norm_backward", "adacomp_relative_buckets",
    "adacomp_bias_softmax_workspace_bytes", "adacomp_bias_softmax_forward", "adacomp_bias_softmax_backward",
]

NORM_COLS_MAX = 32768
BIAS_DISTANCE_MAX = 2048

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_u32, _i32, _u64, _i64, _f32, _vp, _sz = (ctypes.c_uint32, ctypes.c_int32, ctypes.c_uint64, ctypes.c_int64, ctypes.c_float,
                                          ctypes.c_void_p, ctypes.c_size_t)


class _Dropout(ctypes.Structure):
    _fields_ = [("p", _f32), ("reserved", _u32), ("seed", _u64), ("stream", _u64), ("step", _vp)]


class _Norm(ctypes.Structure):
    _fields_ = [("rows", _u64), ("cols", _u32), ("dtype", _u32), ("x_stride", _u64), ("residual_stride", _u64), ("z_stride", _u64),
                ("y_stride", _u64), ("dy_stride", _u64), ("dz_add_stride", _u64), ("dz_stride", _u64), ("dx_stride", _u64)]


class _View(ctypes.Structure):
    _fields_ = [("data", _vp), ("batch_stride", _i64), ("head_stride", _i64), ("row_stride", _i64)]


class _BiasSoftmax(ctypes.Structure):
    _fields_ = [("batch", _u32), ("heads", _u32), ("queries", _u32), ("keys", _u32), ("dtype", _u32), ("causal", _u32), ("n_buckets", _u32),
                ("max_distance", _u32), ("scale", _f32), ("query_start", _i32), ("query_starts", _vp), ("key_lengths", _vp),
                ("table", _vp), ("map", _vp), ("mask", _View)]


_bound = None


def _lib():
    """The library with the argument types of these calls."""
    global _bound
    if _bound is None:
        L = lib()
        P = ctypes.POINTER
        L.adacomp_dropout.argtypes = [_vp, _vp, _vp, _u64, _u64, _u64, _u64, _u64, _u32, P(_Dropout), _vp]
        L.adacomp_norm_forward.argtypes = [P(_Norm), _vp, _vp, _vp, _vp, _f32, P(_Dropout), _vp, _vp, _vp, _vp, _vp]
        L.adacomp_norm_workspace_bytes.argtypes, L.adacomp_norm_workspace_bytes.restype = [_u64, _u64], _sz
        L.adacomp_norm_backward.argtypes = [P(_Norm), _vp, _vp, _vp, _vp, _vp, _vp, P(_Dropout), _vp, _vp, _vp, _vp, ctypes.c_int, _vp, _sz, _vp]
        L.adacomp_relative_buckets.argtypes = [_u32, _u32, ctypes.c_int, _vp]
        L.adacomp_bias_softmax_workspace_bytes.argtypes, L.adacomp_bias_softmax_workspace_bytes.restype = [_u32] * 5, _sz
        L.adacomp_bias_softmax_forward.argtypes = [P(_BiasSoftmax), P(_View), P(_View), _vp, P(_Dropout), _vp, _sz, _vp]
        L.adacomp_bias_softmax_backward.argtypes = [P(_BiasSoftmax), P(_View), _vp, P(_View), P(_Dropout), P(_View), _vp, ctypes.c_int, _vp, _sz, _vp]
        _bound = L
    return _bound


def _refuse(what):
    raise AdacompError(EINVAL, what)


def _stream_of(t):
    device = t.get_device()
    if device < 0 or device != torch.cuda.current_device():
        _refuse("tensors are on the current GPU (there is no CPU path)")
    return torch._C._cuda_getCurrentRawStream(device)   # torch.cuda.current_stream(), without an object around it: 1 us less


def _rows(t, like, what):
    """(address, row stride) of a tensor of like's shape, type and device, seen as rows of its last dimension."""
    if t is None:
        return None, 0
    if t is not like and (t.shape != like.shape or t.dtype != like.dtype or t.get_device() != like.get_device()):
        _refuse(f"{what}: {tuple(t.shape)} {t.dtype} on {t.device} beside {tuple(like.shape)} {like.dtype} on {like.device}")
    if t.is_contiguous():
        return t.data_ptr(), t.shape[-1]
    shape, stride = t.shape, t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        _refuse(f"{what}: the last dimension is not contiguous")
    row, expect = None, 0
    for n, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if row is None:
            row = s
        elif s != expect:
            _refuse(f"{what}: its rows have no single stride")
        expect = s * n
    return t.data_ptr(), shape[-1] if row is None else row


def _vector(t, n, like, what):
    """Address of a contiguous float32 tensor of n values."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != like.get_device():
        _refuse(f"{what}: {n} contiguous float32 values on {like.device} are wanted, it is {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _shape_of(x, what):
    if x.dtype not in _DTYPES:
        _refuse(f"{what}: {x.dtype} is not one of float32, bfloat16, float16")
    if x.dim() == 0:
        _refuse(f"{what}: no dimension")
    cols = x.shape[-1]
    return (x.numel() // cols if cols else 0), cols


def _room(workspace, like):
    if not workspace.is_contiguous() or workspace.get_device() != like.get_device():
        _refuse("workspace: a contiguous tensor on the device of the others is wanted")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


class Dropout:
    """What decides which values a call keeps: rate, seed and the number of the call (`stream`, one per layer and training step).
    `step`, an int64 tensor of one value on the GPU, is added to `stream` when the kernel runs, for captured graphs."""

    def __init__(self, p, seed, stream=0, step=None):
        if step is not None and (step.dtype != torch.int64 or step.numel() != 1 or not step.is_cuda):
            _refuse("step: one int64 value on the GPU is wanted")
        self.p, self.seed, self.stream, self.step = float(p), int(seed), int(stream), step
        self._c = _Dropout(self.p, 0, self.seed & (2 ** 64 - 1), self.stream & (2 ** 64 - 1), None if step is None else step.data_ptr())
        self._ref = ctypes.byref(self._c)


def _drop(dropout, like):
    if dropout is None:
        return None
    if dropout.step is not None and dropout.step.get_device() != like.get_device():
        _refuse("step is on another device")
    return dropout._ref


def adacomp_dropout(x, y, dropout, residual=None):
    """y = D(x), or residual + D(x).  The backward pass is the same call on the gradient."""
    L = _lib()
    rows, cols = _shape_of(x, "x")
    px, sx = _rows(x, x, "x")
    py, sy = _rows(y, x, "y")
    pr, sr = _rows(residual, x, "residual")
    if dropout is None:
        _refuse("dropout is missing")
    _check(L.adacomp_dropout(px, pr, py, rows, cols, sx, sr, sy, _DTYPES[x.dtype], _drop(dropout, x), _stream_of(x)))


def adacomp_norm_forward(x, gamma, beta, y, residual=None, dropout=None, z=None, mean=None, rstd=None, eps=1e-5):
    """z = [residual +] D(x), y = layer norm of z over the last dimension; z, mean and rstd are written where they are given."""
    L = _lib()
    rows, cols = _shape_of(x, "x")
    px, sx = _rows(x, x, "x")
    py, sy = _rows(y, x, "y")
    pr, sr = _rows(residual, x, "residual")
    pz, sz = _rows(z, x, "z")
    norm = _Norm(rows, cols, _DTYPES[x.dtype], sx, sr, sz, sy)
    _check(L.adacomp_norm_forward(ctypes.byref(norm), px, pr, _vector(gamma, cols, x, "gamma"), _vector(beta, cols, x, "beta"), eps, _drop(dropout, x),
                                  pz, py, _vector(mean, rows, x, "mean"), _vector(rstd, rows, x, "rstd"), _stream_of(x)))


def adacomp_norm_workspace_bytes(rows, cols) -> int:
    return int(_lib().adacomp_norm_workspace_bytes(int(rows), int(cols)))


def adacomp_norm_backward(dy, z, mean, rstd, gamma, dz, dgamma, dbeta, workspace, dz_add=None, dropout=None, dx=None, accumulate=False):
    """dz (the gradient of z and of the residual), dx = D(dz), and dgamma, dbeta summed over all rows: overwritten, or with
    accumulate added to.  dgamma and dbeta may be parts of the flat gradient, or None."""
    L = _lib()
    rows, cols = _shape_of(dy, "dy")
    pdy, sdy = _rows(dy, dy, "dy")
    pz, sz = _rows(z, dy, "z")
    pa, sa = _rows(dz_add, dy, "dz_add")
    pdz, sdz = _rows(dz, dy, "dz")
    pdx, sdx = _rows(dx, dy, "dx")
    pw, nw = _room(workspace, dy)
    norm = _Norm(rows, cols, _DTYPES[dy.dtype], 0, 0, sz, 0, sdy, sa, sdz, sdx)
    _check(L.adacomp_norm_backward(ctypes.byref(norm), pdy, pa, pz, _vector(mean, rows, dy, "mean"), _vector(rstd, rows, dy, "rstd"),
                                   _vector(gamma, cols, dy, "gamma"), _drop(dropout, dy), pdz, pdx, _vector(dgamma, cols, dy, "dgamma"),
                                   _vector(dbeta, cols, dy, "dbeta"), 1 if accumulate else 0, pw, nw, _stream_of(dy)))


def adacomp_relative_buckets(n_buckets, max_distance, both_directions):
    """The usual logarithmic map of distances key - query in -max_distance .. max_distance to buckets, as an int32 numpy array."""
    out = np.zeros(2 * int(max_distance) + 1, np.int32)
    _check(_lib().adacomp_relative_buckets(int(n_buckets), int(max_distance), 1 if both_directions else 0, out.ctypes.data))
    return out


class RelativeBias:
    """A learned bias by buckets of distance: `table` [n_buckets, heads] float32 (it may be a part of the flat weights) and `map`, an int32
    tensor of 2 * max_distance + 1 buckets on the GPU."""

    def __init__(self, table, map):
        if table.dim() != 2 or table.dtype != torch.float32 or not table.is_contiguous():
            _refuse("table: a contiguous float32 tensor [n_buckets, heads] is wanted")
        if map.dim() != 1 or map.dtype != torch.int32 or not map.is_contiguous() or map.numel() % 2 == 0 or map.get_device() != table.get_device():
            _refuse("map: an int32 tensor of 2 * max_distance + 1 values beside the table is wanted")
        self.table, self.map = table, map
        self.n_buckets, self.heads = table.shape
        self.max_distance = map.numel() // 2


def _view(t, like, what):
    if t is not like and (t.shape != like.shape or t.dtype != like.dtype or t.get_device() != like.get_device()):
        _refuse(f"{what}: {tuple(t.shape)} {t.dtype} on {t.device} beside {tuple(like.shape)} {like.dtype} on {like.device}")
    s = t.stride()
    if s[3] != 1 and t.shape[3] > 1:
        _refuse(f"{what}: the last dimension is not contiguous")
    return _View(t.data_ptr(), s[0], s[1], s[2])


def _per_sequence(t, batch, like, what):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.numel() != batch or not t.is_contiguous() or t.get_device() != like.get_device():
        _refuse(f"{what}: an int32 value for each of {batch} sequences is wanted")
    return t.data_ptr()


def _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask):
    if scores.dim() != 4 or scores.dtype not in _DTYPES:
        _refuse("scores: [batch, heads, queries, keys] of float32, bfloat16 or float16 is wanted")
    b, h, q, k = scores.shape
    if bias.heads != h or bias.table.get_device() != scores.get_device():
        _refuse(f"the bias is one of {bias.heads} heads on {bias.table.device}, the scores have {h} on {scores.device}")
    view = _View()
    if mask is not None:
        if mask.dtype not in (torch.uint8, torch.bool) or mask.dim() != 4 or mask.get_device() != scores.get_device():
            _refuse("mask: a uint8 or bool tensor of 4 dimensions is wanted")
        mask = mask.expand(b, h, q, k)   # no copy: strides of 0
        s = mask.stride()
        if s[3] != 1 and k > 1:
            _refuse("mask: its last dimension is contiguous and as long as the scores'")
        view = _View(mask.data_ptr(), s[0], s[1], s[2])
    return _BiasSoftmax(b, h, q, k, _DTYPES[scores.dtype], 1 if causal else 0, bias.n_buckets, bias.max_distance, scale, int(query_start),
                        _per_sequence(query_starts, b, scores, "query_starts"), _per_sequence(key_lengths, b, scores, "key_lengths"),
                        bias.table.data_ptr(), bias.map.data_ptr(), view)


def adacomp_bias_softmax_workspace_bytes(batch, heads, queries, keys, max_distance) -> int:
    return int(_lib().adacomp_bias_softmax_workspace_bytes(int(batch), int(heads), int(queries), int(keys), int(max_distance)))


def adacomp_bias_softmax_forward(scores, bias, probs, workspace, lse=None, scale=1.0, causal=False, query_start=0, query_starts=None,
                                 key_lengths=None, mask=None, dropout=None):
    """probs = D(softmax(scale * scores + bias)) over the admitted keys (see adacomp_layers.h); lse [batch, heads, queries], for the
    backward pass, is written if it is given.  The mask may have dimensions of 1 before the last."""
    L = _lib()
    op = _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask)
    pw, nw = _room(workspace, scores)
    rows = op.batch * op.heads * op.queries
    _check(L.adacomp_bias_softmax_forward(ctypes.byref(op), ctypes.byref(_view(scores, scores, "scores")), ctypes.byref(_view(probs, scores, "probs")),
                                          _vector(lse, rows, scores, "lse"), _drop(dropout, scores), pw, nw, _stream_of(scores)))


def adacomp_bias_softmax_backward(scores, bias, lse, dprobs, dscores, dtable, workspace, scale=1.0, causal=False, query_start=0, query_starts=None,
                                  key_lengths=None, mask=None, dropout=None, accumulate=False):
    """dscores and dtable (a part of the flat gradient, or None) from dprobs, with the other arguments as in the forward pass."""
    L = _lib()
    op = _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask)
    pw, nw = _room(workspace, scores)
    rows = op.batch * op.heads * op.queries
    _check(L.adacomp_bias_softmax_backward(ctypes.byref(op), ctypes.byref(_view(scores, scores, "scores")), _vector(lse, rows, scores, "lse"),
                                           ctypes.byref(_view(dprobs, scores, "dprobs")), _drop(dropout, scores),
                                           ctypes.byref(_view(dscores, scores, "dscores")), _vector(dtable, op.n_buckets * op.heads, scores, "dtable"),
                                           1 if accumulate else 0, pw, nw, _stream_of(scores)))

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


_bound = None   # the library, once it has the argument types below


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


_current_device = torch._C._cuda_getDevice          # torch.cuda.current_device() and torch.cuda.current_stream() without an object
_current_stream = torch._C._cuda_getCurrentRawStream   # and a look at the module's state around them: 1 us less, of 8 in all


def _in_32_bits(x, what):
    """x, a size or number that the library takes as an unsigned 32-bit one: ctypes would cut off what is above."""
    if not 0 <= x < 2 ** 32:
        _refuse(f"{what}: {x} is not a number of 32 bits")
    return x


def _device_of(x):
    """The GPU that x and every other tensor of the call have to be on."""
    device = x.get_device()
    if device < 0 or device != _current_device():
        _refuse("tensors are on the current GPU (there is no CPU path)")
    return device


def _unlike(t, shape, dtype, what):
    _refuse(f"{what}: {tuple(t.shape)} {t.dtype} on {t.device} where {tuple(shape)} {dtype} on the device of the first tensor is wanted")


def _rows(t, shape, dtype, device, what):
    """(address, row stride) of a tensor of the given shape, type and device, seen as rows of its last dimension."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _unlike(t, shape, dtype, what)
    if t.is_contiguous():
        return t.data_ptr(), shape[-1]
    stride = t.stride()
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


def _vector(t, n, device, what):
    """Address of a contiguous float32 tensor of n values."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        _unlike(t, (n,), "contiguous torch.float32", what)
    return t.data_ptr()


def _shape_of(x, what):
    """(shape, type, its number, rows, columns)"""
    shape, dtype = x.shape, x.dtype
    number = _DTYPES.get(dtype)
    if number is None:
        _refuse(f"{what}: {dtype} is not one of float32, bfloat16, float16")
    if not shape:
        _refuse(f"{what}: no dimension")
    cols = shape[-1]
    return shape, dtype, number, (x.numel() // cols if cols else 0), cols


def _room(workspace, device):
    if not workspace.is_contiguous() or workspace.get_device() != device:
        _refuse("workspace: a contiguous tensor on the device of the others is wanted")
    return workspace.data_ptr(), workspace.nbytes


class Dropout:
    """What decides which values a call keeps: rate, seed and the number of the call (`stream`, one per layer and training step).
    `step`, an int64 tensor of one value on the GPU, is added to `stream` when the kernel runs, for captured graphs.
    The attributes can be set; calls from then on use what they are."""

    def __init__(self, p, seed, stream=0, step=None):
        self._c = _Dropout()
        self._ref = ctypes.byref(self._c)
        self.p, self.seed, self.stream, self.step = p, seed, stream, step

    @property
    def p(self):
        return self._p

    @p.setter
    def p(self, p):
        self._p = self._c.p = float(p)

    @property
    def seed(self):
        return self._seed

    @seed.setter
    def seed(self, seed):
        self._seed = int(seed)
        self._c.seed = self._seed & (2 ** 64 - 1)

    @property
    def stream(self):
        return self._stream

    @stream.setter
    def stream(self, stream):
        self._stream = int(stream)
        self._c.stream = self._stream & (2 ** 64 - 1)

    @property
    def step(self):
        return self._step

    @step.setter
    def step(self, step):
        if step is not None and (step.dtype != torch.int64 or step.numel() != 1 or not step.is_cuda):
            _refuse("step: one int64 value on the GPU is wanted")
        self._step = step
        self._c.step = None if step is None else step.data_ptr()


def _drop(dropout, device):
    if dropout is None:
        return None
    if dropout._step is not None and dropout._step.get_device() != device:
        _refuse("step is on another device")
    return dropout._ref


def adacomp_dropout(x, y, dropout, residual=None):
    """y = D(x), or residual + D(x).  The backward pass is the same call on the gradient."""
    L = _bound or _lib()
    shape, dtype, number, rows, cols = _shape_of(x, "x")
    dev = _device_of(x)
    px, sx = _rows(x, shape, dtype, dev, "x")
    py, sy = _rows(y, shape, dtype, dev, "y")
    pr, sr = _rows(residual, shape, dtype, dev, "residual")
    if dropout is None:
        _refuse("dropout is missing")
    rc = L.adacomp_dropout(px, pr, py, rows, cols, sx, sr, sy, number, _drop(dropout, dev), _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_norm_forward(x, gamma, beta, y, residual=None, dropout=None, z=None, mean=None, rstd=None, eps=1e-5):
    """z = [residual +] D(x), y = layer norm of z over the last dimension; z, mean and rstd are written where they are given."""
    L = _bound or _lib()
    shape, dtype, number, rows, cols = _shape_of(x, "x")
    dev = _device_of(x)
    px, sx = _rows(x, shape, dtype, dev, "x")
    py, sy = _rows(y, shape, dtype, dev, "y")
    pr, sr = _rows(residual, shape, dtype, dev, "residual")
    pz, sz = _rows(z, shape, dtype, dev, "z")
    if cols >> 32:
        _in_32_bits(cols, "columns")
    norm = _Norm(rows, cols, number, sx, sr, sz, sy)
    rc = L.adacomp_norm_forward(norm, px, pr, _vector(gamma, cols, dev, "gamma"), _vector(beta, cols, dev, "beta"), eps, _drop(dropout, dev), pz, py,
                                _vector(mean, rows, dev, "mean"), _vector(rstd, rows, dev, "rstd"), _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_norm_workspace_bytes(rows, cols) -> int:
    rows, cols = int(rows), int(cols)
    return int(_lib().adacomp_norm_workspace_bytes(rows, cols)) if 0 <= rows < 2 ** 32 and 0 <= cols < 2 ** 32 else 0


def adacomp_norm_backward(dy, z, mean, rstd, gamma, dz, dgamma, dbeta, workspace, dz_add=None, dropout=None, dx=None, accumulate=False):
    """dz (the gradient of z and of the residual), dx = D(dz), and dgamma, dbeta summed over all rows: overwritten, or with
    accumulate added to.  dgamma and dbeta may be parts of the flat gradient, or None."""
    L = _bound or _lib()
    shape, dtype, number, rows, cols = _shape_of(dy, "dy")
    dev = _device_of(dy)
    pdy, sdy = _rows(dy, shape, dtype, dev, "dy")
    pz, sz = _rows(z, shape, dtype, dev, "z")
    pa, sa = _rows(dz_add, shape, dtype, dev, "dz_add")
    pdz, sdz = _rows(dz, shape, dtype, dev, "dz")
    pdx, sdx = _rows(dx, shape, dtype, dev, "dx")
    pw, nw = _room(workspace, dev)
    if cols >> 32:
        _in_32_bits(cols, "columns")
    norm = _Norm(rows, cols, number, 0, 0, sz, 0, sdy, sa, sdz, sdx)
    rc = L.adacomp_norm_backward(norm, pdy, pa, pz, _vector(mean, rows, dev, "mean"), _vector(rstd, rows, dev, "rstd"), _vector(gamma, cols, dev, "gamma"),
                                 _drop(dropout, dev), pdz, pdx, _vector(dgamma, cols, dev, "dgamma"), _vector(dbeta, cols, dev, "dbeta"),
                                 1 if accumulate else 0, pw, nw, _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_relative_buckets(n_buckets, max_distance, both_directions):
    """The usual logarithmic map of distances key - query in -max_distance .. max_distance to buckets, as an int32 numpy array."""
    n_buckets, max_distance = _in_32_bits(int(n_buckets), "n_buckets"), int(max_distance)
    if not 1 <= max_distance <= BIAS_DISTANCE_MAX:
        _refuse(f"max_distance: {max_distance} is not one of 1 .. {BIAS_DISTANCE_MAX}")
    out = np.zeros(2 * max_distance + 1, np.int32)
    _check(_lib().adacomp_relative_buckets(n_buckets, max_distance, 1 if both_directions else 0, out.ctypes.data))
    return out


class RelativeBias:
    """A learned bias by buckets of distance: `table` [n_buckets, heads] float32 (it may be a part of the flat weights) and `map`, an int32
    tensor of 2 * max_distance + 1 buckets on the GPU.  Both can be set; the sizes are theirs."""

    def __init__(self, table, map):
        self.table, self.map = table, map

    n_buckets = property(lambda self: self._n_buckets)
    heads = property(lambda self: self._heads)
    max_distance = property(lambda self: self._max_distance)

    @property
    def table(self):
        return self._table

    @table.setter
    def table(self, table):
        if table.dim() != 2 or table.dtype != torch.float32 or not table.is_contiguous():
            _refuse("table: a contiguous float32 tensor [n_buckets, heads] is wanted")
        self._n_buckets, self._heads = _in_32_bits(table.shape[0], "buckets"), table.shape[1]
        self._table = table

    @property
    def map(self):
        return self._map

    @map.setter
    def map(self, map):
        if map.dim() != 1 or map.dtype != torch.int32 or not map.is_contiguous() or map.numel() % 2 == 0 or map.get_device() != self._table.get_device():
            _refuse("map: an int32 tensor of 2 * max_distance + 1 values beside the table is wanted")
        self._max_distance = _in_32_bits(map.numel() // 2, "max_distance")
        self._map = map


def _view(t, shape, dtype, device, what):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _unlike(t, shape, dtype, what)
    b, h, q, k = t.stride()
    if k != 1 and shape[3] > 1:
        _refuse(f"{what}: the last dimension is not contiguous")
    return _View(t.data_ptr(), b, h, q)


def _per_sequence(t, batch, device, what):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() != batch or not t.is_contiguous() or t.get_device() != device:
        _unlike(t, (batch,), "contiguous torch.int32", what)
    return t.data_ptr()


def _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask):
    """(the operator, shape, type and device of its tensors, rows)"""
    shape, dtype = scores.shape, scores.dtype
    number = _DTYPES.get(dtype)
    if len(shape) != 4 or number is None:
        _refuse("scores: [batch, heads, queries, keys] of float32, bfloat16 or float16 is wanted")
    dev = _device_of(scores)
    b, h, q, k = shape
    if bias._heads != h or bias._table.get_device() != dev or bias._map.get_device() != dev:
        _refuse(f"the bias is one of {bias._heads} heads on {bias._table.device} (its map on {bias._map.device}), the scores have {h} on {scores.device}")
    if (b | h | q | k) >> 32 or query_start and not -2 ** 31 <= query_start < 2 ** 31:   # ctypes would cut off what is above
        _refuse(f"sizes {tuple(shape)}, query_start {query_start}: not all are numbers of 32 bits")
    view = _NO_VIEW
    if mask is not None:
        if mask.dtype not in (torch.uint8, torch.bool) or mask.dim() != 4 or mask.get_device() != dev:
            _refuse("mask: a uint8 or bool tensor of 4 dimensions is wanted")
        if any(n != 1 and n != m for n, m in zip(mask.shape, shape)):
            _refuse(f"mask: {tuple(mask.shape)} beside scores of {tuple(shape)}")
        mask = mask.expand(b, h, q, k)   # no copy: strides of 0
        s = mask.stride()
        if s[3] != 1 and k > 1:
            _refuse("mask: its last dimension is contiguous and as long as the scores'")
        view = _View(mask.data_ptr(), s[0], s[1], s[2])
    op = _BiasSoftmax(b, h, q, k, number, 1 if causal else 0, bias._n_buckets, bias._max_distance, scale, query_start,
                      _per_sequence(query_starts, b, dev, "query_starts"), _per_sequence(key_lengths, b, dev, "key_lengths"),
                      bias._table.data_ptr(), bias._map.data_ptr(), view)
    return op, shape, dtype, dev, b * h * q


_NO_VIEW = _View()


def adacomp_bias_softmax_workspace_bytes(batch, heads, queries, keys, max_distance) -> int:
    sizes = [int(n) for n in (batch, heads, queries, keys, max_distance)]
    return int(_lib().adacomp_bias_softmax_workspace_bytes(*sizes)) if all(0 <= n < 2 ** 32 for n in sizes) else 0


def adacomp_bias_softmax_forward(scores, bias, probs, workspace, lse=None, scale=1.0, causal=False, query_start=0, query_starts=None,
                                 key_lengths=None, mask=None, dropout=None):
    """probs = D(softmax(scale * scores + bias)) over the admitted keys (see adacomp_layers.h); lse [batch, heads, queries], for the
    backward pass, is written if it is given.  The mask may have dimensions of 1 before the last."""
    L = _bound or _lib()
    op, shape, dtype, dev, rows = _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask)
    pw, nw = _room(workspace, dev)
    rc = L.adacomp_bias_softmax_forward(op, _view(scores, shape, dtype, dev, "scores"), _view(probs, shape, dtype, dev, "probs"),
                                        _vector(lse, rows, dev, "lse"), _drop(dropout, dev), pw, nw, _current_stream(dev))
    if rc:
        _check(rc)


def adacomp_bias_softmax_backward(scores, bias, lse, dprobs, dscores, dtable, workspace, scale=1.0, causal=False, query_start=0, query_starts=None,
                                  key_lengths=None, mask=None, dropout=None, accumulate=False):
    """dscores and dtable (a part of the flat gradient, or None) from dprobs, with the other arguments as in the forward pass."""
    L = _bound or _lib()
    op, shape, dtype, dev, rows = _bias_softmax(scores, bias, scale, causal, query_start, query_starts, key_lengths, mask)
    pw, nw = _room(workspace, dev)
    rc = L.adacomp_bias_softmax_backward(op, _view(scores, shape, dtype, dev, "scores"), _vector(lse, rows, dev, "lse"),
                                         _view(dprobs, shape, dtype, dev, "dprobs"), _drop(dropout, dev), _view(dscores, shape, dtype, dev, "dscores"),
                                         _vector(dtable, bias._n_buckets * bias._heads, dev, "dtable"), 1 if accumulate else 0, pw, nw, _current_stream(dev))
    if rc:
        _check(rc)

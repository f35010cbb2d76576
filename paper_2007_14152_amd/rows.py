"""The ends of a mixture of networks (the second half of include/spdnn.h) on torch tensors.

Argument marshalling only, as in the package's __init__: torch allocates the outputs and names the stream, the HIP kernels
do the rest.  Gradients are calls of their own: nothing is recorded for automatic ones, and a call warns where an input asks for one
(outside torch.no_grad()).  Every call enqueues on the current
stream of its tensors' device and returns without waiting.  Rows may have any stride between them, their elements are adjacent;
what the library refuses raises SpdnnError.
"""
from __future__ import annotations

import ctypes
import functools
import warnings

import torch

from . import (SPDNN_BF16, SPDNN_EINVAL, SPDNN_F16, SPDNN_F32, SPDNN_I32, SPDNN_I64, SPDNN_SIGMOID, SPDNN_SOFTMAX, SpdnnError,
               _check, lib)

_TYPES = {torch.float32: SPDNN_F32, torch.bfloat16: SPDNN_BF16, torch.float16: SPDNN_F16}
_IDS = {torch.int32: SPDNN_I32, torch.int64: SPDNN_I64}
_SCORES = {"softmax": SPDNN_SOFTMAX, "sigmoid": SPDNN_SIGMOID}


def _refuse(text, *args):
    raise SpdnnError(SPDNN_EINVAL, text % args)


def _unrecorded(name, level=3):
    """For a call of which an input asks for a gradient."""
    if torch.is_grad_enabled():
        warnings.warn("%s records no gradient for its inputs: call the gradient's operator, or wrap the call in torch.no_grad()" % name,
                      stacklevel=level)


_MOST = 2 ** 31 - 1  # the library's sizes are of 32 bits; ctypes would pass on the last 32 of more without a word


def _fits(name, *sizes):
    for size in sizes:
        if not -_MOST <= size <= _MOST:
            _refuse("%s: a size of %d, at most %d", name, size, _MOST)


def _type(dtype, name):
    code = _TYPES.get(dtype)
    if code is None:
        _refuse("%s: float32, bfloat16 or float16, not %s", name, dtype)
    return code


def _rows(t, name, device=None, shape=None):
    """(type, stride) of a matrix of rows."""
    size = t.shape
    if len(size) != 2 or not t.is_cuda:
        _refuse("%s: a matrix in GPU memory, not %s on %s", name, tuple(size), t.device)
    if device is not None and t.device != device:
        _refuse("%s is on %s, not on %s", name, t.device, device)
    if shape is not None and size != shape:
        _refuse("%s: %s, not %s", name, shape, tuple(size))
    if size[0] > _MOST or size[1] > _MOST:
        _fits(name, *size)
    stride, step = t.stride()
    if step != 1 and size[1] > 1:
        _refuse("%s: the elements of a row must be adjacent", name)
    code = _TYPES.get(t.dtype)
    if code is None:
        _type(t.dtype, name)
    return code, stride if size[0] > 1 else max(stride, size[1])


def _array(t, name, dtypes, device, shape):
    """Address of a contiguous array, 0 for None."""
    if t is None:
        return 0
    if t.dtype not in dtypes or t.device != device or t.shape != shape or not t.is_contiguous():
        _refuse("%s: a contiguous %s of %s on %s, not %s of %s on %s", name, shape, dtypes[0], device, tuple(t.shape), t.dtype, t.device)
    return t.data_ptr()


def _pairs(t, name):
    """(rows, k) of what stands for every pair of a row and a slot."""
    if t.dim() != 2:
        _refuse("%s: a matrix, not %s", name, tuple(t.shape))
    rows, k = t.shape
    if rows > _MOST or k > _MOST:
        _fits(name, rows, k)
    return rows, k


_F32 = (torch.float32,)
_I32 = (torch.int32,)
_BYTES = (torch.bool, torch.uint8)

# The number of the current device, and the raw handle of a device's current stream.  (torch.cuda.current_stream makes an object
# around it first, which takes 1.9 us; the smallest call there is takes 4.5.)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


@functools.lru_cache(maxsize=64)
def _work_bytes(name, *sizes):
    _fits(name, *sizes)
    need = ctypes.c_size_t()
    _check(getattr(lib(), name)(*sizes, ctypes.byref(need)))
    return need.value


def embed(table, ids, scale=1.0, dtype=None):
    """scale * table[ids], rows of zeros for ids outside the table (padding): [*ids.shape, width] of dtype (the table's).

    table: float32, bfloat16 or float16 [vocab, width]; ids: int32 or int64 of any shape."""
    ttype, tstride = _rows(table, "table")
    vocab, width = table.shape
    otype = ttype if dtype is None else _type(dtype, "dtype")
    dev = table.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return embed(table, ids, scale, dtype)
    if table.requires_grad:
        _unrecorded("embed")
    if ids.dtype not in _IDS or ids.device != dev:
        _refuse("ids: int32 or int64 on %s, not %s on %s", dev, ids.dtype, ids.device)
    n = ids.numel()
    if n > _MOST:
        _fits("ids", n)
    ids = ids.contiguous()
    out = table.new_empty((*ids.shape, width), dtype=dtype)
    _check(lib().spdnn_embed(table.data_ptr(), ttype, vocab, width, tstride, ids.data_ptr(), _IDS[ids.dtype], n,
                             scale, out.data_ptr(), otype, width, _stream(dev.index)))
    return out


def embed_grad(dout, ids, vocab, scale=1.0, dtype=torch.float32, out=None):
    """Gradient of embed's table, [vocab, width]: scale * the sum of dout's rows of each id.

    dout: [n, width] rows (or [*ids.shape, width], contiguous); ids: int32 or int64, n of them.  out: a table of gradients
    to which the sums are added in place (its type and size are then taken from it; rows of ids that do not occur stay
    untouched)."""
    if dout.dim() != 2:
        dout = dout.reshape(-1, dout.shape[-1])
    itype, dstride = _rows(dout, "dout")
    n, width = dout.shape
    dev = dout.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return embed_grad(dout, ids, vocab, scale, dtype, out)
    if dout.requires_grad or out is not None and out.requires_grad:
        _unrecorded("embed_grad")
    if ids.dtype not in _IDS or ids.device != dev or ids.numel() != n:
        _refuse("ids: %d of int32 or int64 on %s, not %d of %s on %s", n, dev, ids.numel(), ids.dtype, ids.device)
    ids = ids.contiguous()
    add = out is not None
    need = _work_bytes("spdnn_embed_grad_bytes", vocab, width, n)
    if not add:
        _type(dtype, "dtype")
        out = dout.new_empty((vocab, width), dtype=dtype)
    otype, ostride = _rows(out, "out", dev, (vocab, width))
    work = dout.new_empty(need, dtype=torch.uint8) if need else None
    _check(lib().spdnn_embed_grad(dout.data_ptr(), itype, dstride, ids.data_ptr(), _IDS[ids.dtype], n, vocab, width, scale, add,
                                  out.data_ptr(), otype, ostride, work.data_ptr() if need else 0, need, _stream(dev.index)))
    if add:
        torch.autograd.graph.increment_version(out)  # changed in place: what an automatic gradient has kept of it is stale
    return out


def _score(score):
    if score not in _SCORES:
        _refuse("score: softmax or sigmoid, not %r", score)
    return _SCORES[score]


def route(logits, k, bias=None, keep=None, score="softmax", normalise=True, scale=1.0):
    """(chosen int32 [rows, k], weight float32 [rows, k]): the k experts of each row with the largest logits (plus bias,
    which only the choice sees), and their weights; -1 and 0 where a row has no expert left.

    bias: float32 [experts], on the logit (not on its sigmoid, where some routers have it); keep: bool [rows], False for rows that go to no expert (padding)."""
    ltype, stride = _rows(logits, "logits")
    rows, experts = logits.shape
    dev = logits.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return route(logits, k, bias, keep, score, normalise, scale)
    if logits.requires_grad or bias is not None and bias.requires_grad:
        _unrecorded("route")
    if not -_MOST <= k <= _MOST:
        _fits("k", k)
    bp = _array(bias, "bias", _F32, dev, (experts,))
    kp = _array(keep, "keep", _BYTES, dev, (rows,))
    chosen = logits.new_empty((rows, max(k, 0)), dtype=torch.int32)
    weight = logits.new_empty((rows, max(k, 0)), dtype=torch.float32)
    _check(lib().spdnn_route(logits.data_ptr(), ltype, stride, rows, experts, k, bp, kp, _score(score), normalise, scale,
                             chosen.data_ptr(), weight.data_ptr(), _stream(dev.index)))
    return chosen, weight


def route_grad(dweight, logits, chosen, bias=None, score="softmax", normalise=True, scale=1.0):
    """Gradient of route's weights with respect to the logits, of the logits' type; chosen, bias, score, normalise and scale
    as they were there."""
    ltype, stride = _rows(logits, "logits")
    rows, experts = logits.shape
    dev = logits.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return route_grad(dweight, logits, chosen, bias, score, normalise, scale)
    if logits.requires_grad or dweight.requires_grad or bias is not None and bias.requires_grad:
        _unrecorded("route_grad")
    k = _pairs(chosen, "chosen")[1]
    bp = _array(bias, "bias", _F32, dev, (experts,))
    cp = _array(chosen, "chosen", _I32, dev, (rows, k))
    wp = _array(dweight, "dweight", _F32, dev, (rows, k))
    out = logits.new_empty((rows, experts))
    _check(lib().spdnn_route_grad(wp, logits.data_ptr(), ltype, stride, cp, rows, experts, k, bp, _score(score), normalise,
                                  scale, out.data_ptr(), experts, _stream(dev.index)))
    return out


def dispatch(x, chosen, experts):
    """(xs [rows * k, width], offsets int32 [experts + 1], place int32 [rows, k]): x's rows sorted by expert, once for each
    expert they go to.  Expert e has the rows offsets[e] .. offsets[e + 1] of xs; row t's copy for its slot j is row
    place[t, j] of xs, -1 if chosen[t, j] is no expert; rows of xs without a pair are zero."""
    xtype, xstride = _rows(x, "x")
    rows, width = x.shape
    dev = x.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return dispatch(x, chosen, experts)
    if x.requires_grad:
        _unrecorded("dispatch")
    k = _pairs(chosen, "chosen")[1]
    cp = _array(chosen, "chosen", _I32, dev, (rows, k))
    need = _work_bytes("spdnn_dispatch_bytes", rows, k, experts)
    xs = x.new_empty((rows * k, width))
    offsets = chosen.new_empty(experts + 1)
    place = chosen.new_empty((rows, k))
    work = x.new_empty(need, dtype=torch.uint8) if need else None
    _check(lib().spdnn_dispatch(cp, rows, k, experts, x.data_ptr(), xtype, width, xstride, xs.data_ptr(), width, offsets.data_ptr(),
                                place.data_ptr(), work.data_ptr() if need else 0, need, _stream(dev.index)))
    return xs, offsets, place


def _back(name, ys, place, weight, add):
    ytype, ystride = _rows(ys, "ys")
    dev = ys.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return _back(name, ys, place, weight, add)
    if ys.requires_grad or weight is not None and weight.requires_grad or add is not None and add.requires_grad:
        _unrecorded(name, 4)
    rows, k = _pairs(place, "place")
    width = ys.shape[1]
    if ys.shape[0] != rows * k:
        _refuse("ys: %d rows for %d x %d places", ys.shape[0], rows, k)
    pp = _array(place, "place", _I32, dev, (rows, k))
    wp = _array(weight, "weight", _F32, dev, (rows, k))
    ap, astride = 0, width
    if add is not None:
        atype, astride = _rows(add, "add", dev, (rows, width))
        if atype != ytype:
            _refuse("add: %s, not %s", ys.dtype, add.dtype)
        ap = add.data_ptr()
    out = ys.new_empty((rows, width))
    _check(lib().spdnn_combine(ys.data_ptr(), ytype, width, ystride, pp, wp, rows, k, ap, astride, out.data_ptr(), width,
                               _stream(dev.index)))
    return out


def combine(ys, place, weight=None, add=None):
    """add + the sum over j of weight[:, j] * ys[place[:, j]]: the way back from dispatch's order, [rows, width].

    ys: [rows * k, width]; weight: float32 [rows, k], ones if None; add: [rows, width] of ys's type (a residual), zeros if
    None.  Slots whose place is -1 are left out."""
    return _back("combine", ys, place, weight, add)


def dispatch_grad(dxs, place):
    """Gradient of dispatch: the sum of the gradients of a row's copies."""
    return _back("dispatch_grad", dxs, place, None, None)


def combine_grad(dout, ys, place, weight, offsets):
    """(dys, dweight): gradients of combine with respect to ys and weight (that of add is dout).  offsets as dispatch gave
    them: rows of dys without a pair are zero."""
    ytype, ystride = _rows(ys, "ys")
    dev = ys.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return combine_grad(dout, ys, place, weight, offsets)
    if dout.requires_grad or ys.requires_grad or weight is not None and weight.requires_grad:
        _unrecorded("combine_grad")
    rows, k = _pairs(place, "place")
    width = ys.shape[1]
    if ys.shape[0] != rows * k:
        _refuse("ys: %d rows for %d x %d places", ys.shape[0], rows, k)
    gtype, gstride = _rows(dout, "dout", dev, (rows, width))
    if gtype != ytype:
        _refuse("dout: %s, not %s", ys.dtype, dout.dtype)
    pp = _array(place, "place", _I32, dev, (rows, k))
    if weight is None:
        _refuse("weight is None")
    wp = _array(weight, "weight", _F32, dev, (rows, k))
    if offsets.dim() != 1 or offsets.shape[0] < 2:
        _refuse("offsets: one per expert and the end, not %s", tuple(offsets.shape))
    op = _array(offsets, "offsets", _I32, dev, tuple(offsets.shape))
    dys = ys.new_empty((rows * k, width))
    dweight = weight.new_empty((rows, k))
    _check(lib().spdnn_combine_grad(dout.data_ptr(), ytype, width, gstride, ys.data_ptr(), ystride, pp, wp,
                                    op + 4 * (offsets.shape[0] - 1), rows, k, dys.data_ptr(), width, dweight.data_ptr(),
                                    _stream(dev.index)))
    return dys, dweight

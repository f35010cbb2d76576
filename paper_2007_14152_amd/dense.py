"""Dense products and layer norm around a mixture of networks (the last part of include/spdnn.h) on torch tensors.

Argument marshalling only, in the manner of rows.py: torch allocates outputs and work memory and names the stream, the HIP
kernels do the rest.  Gradients are calls of their own: nothing is recorded for automatic ones, and a call warns where an input
asks for one (outside torch.no_grad()).  Every call enqueues on the current stream of its tensors' device and returns without
waiting.  Rows may have any stride between them, their elements are adjacent; weights have their columns or their rows adjacent
(the transposed view of a matrix that is stored [out, in] is fine); what the library refuses raises SpdnnError.
"""
from __future__ import annotations

import torch

from . import SPDNN_ACT_CLIP, SPDNN_ACT_GELU, SPDNN_ACT_NONE, SPDNN_ACT_RELU, SPDNN_ACT_SILU, SPDNN_F32, _check, lib
from .rows import _F32, _I32, _MOST, _TYPES, _array, _current, _fits, _refuse, _rows, _stream, _type, _unrecorded, _work_bytes

_ACTS = {None: SPDNN_ACT_NONE, "relu": SPDNN_ACT_RELU, "clip": SPDNN_ACT_CLIP, "gelu": SPDNN_ACT_GELU, "silu": SPDNN_ACT_SILU}


def _act(act):
    code = _ACTS.get(act) if act is None or isinstance(act, str) else None
    if code is None:
        _refuse("act: None, relu, clip, gelu or silu, not %r", act)
    return code


def _weight(t, x, sets):
    """(experts, width, cols, whether stored the other way round, stride, stride between experts) of x's weights."""
    size = t.shape
    if len(size) != 2 + sets:
        _refuse("weight: %s, not %s", "[experts, in, out]" if sets else "[in, out]", tuple(size))
    if t.dtype != x.dtype or t.device != x.device:
        _refuse("weight: %s on %s, not %s on %s", x.dtype, x.device, t.dtype, t.device)
    width, cols = size[-2:]
    if width != x.shape[1]:
        _refuse("weight: %d rows for x of width %d", width, x.shape[1])
    if cols > _MOST or sets and size[0] > _MOST:
        _fits("weight", *size)
    stride, step = t.stride()[-2:]
    transposed = (stride == 1 or width == 1) and (step != 1 or cols == 1)
    if transposed:
        line = step if cols > 1 else max(step, width)
    elif step == 1 or cols == 1:
        line = stride if width > 1 else max(stride, cols)
    else:
        _refuse("weight: neither its rows nor its columns are adjacent (strides %s)", tuple(t.stride()))
    return size[0] if sets else 1, width, cols, transposed, line, t.stride(0) if sets else 0


def _vector(t, name, x, shape):
    """(address, type) of contiguous parameters in x's type or float32."""
    if t is None:
        return 0, SPDNN_F32
    p = _array(t, name, (x.dtype, torch.float32), x.device, shape)
    return p, _TYPES[t.dtype]


def _asks(*tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            return True
    return False


def _offsets(offsets, weight, x):
    if weight.dim() != 3:
        _refuse("weight: [experts, in, out], not %s", tuple(weight.shape))
    return _array(offsets, "offsets", _I32, x.device, (weight.shape[0] + 1,))


def _forward(name, x, offsets, weight, bias, act, add, pre, dtype):
    xtype, xstride = _rows(x, "x")
    dev = x.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return _forward(name, x, offsets, weight, bias, act, add, pre, dtype)
    if _asks(x, weight, bias, add):
        _unrecorded(name, 4)
    sets = offsets is not None
    op = _offsets(offsets, weight, x) if sets else 0
    experts, width, cols, transposed, wstride, estride = _weight(weight, x, sets)
    rows = x.shape[0]
    otype = xtype if dtype is None else _type(dtype, "dtype")
    bp, btype = _vector(bias, "bias", x, (experts, cols) if sets else (cols,))
    ap, astride = 0, cols
    if add is not None:
        atype, astride = _rows(add, "add", dev, (rows, cols))
        if atype != otype:
            _refuse("add: %s, not %s", dtype or x.dtype, add.dtype)
        ap = add.data_ptr()
    act = _act(act)
    need = _work_bytes("spdnn_linear_bytes", rows, width, cols, sets, experts, xtype)
    out = x.new_empty((rows, cols), dtype=dtype)
    before = torch.empty_like(out) if pre else None
    work = x.new_empty(need, dtype=torch.uint8) if need else None
    _check(lib().spdnn_linear(x.data_ptr(), xtype, rows, width, xstride, op, experts, weight.data_ptr(), transposed, wstride, estride, cols,
                              bp, btype, act, ap, astride, out.data_ptr(), otype, cols, before.data_ptr() if pre else 0, cols,
                              work.data_ptr() if need else 0, need, _stream(dev.index)))
    return (out, before) if pre else out


def linear(x, weight, bias=None, act=None, add=None, pre=False, dtype=None):
    """act(x @ weight + bias) + add: [rows, out] of dtype (x's, or float32).

    x: [rows, in]; weight: [in, out] of x's type; bias: [out] of x's type or float32; act: None, "relu", "clip" (to 0 .. 32, as the
    sparse networks do), "gelu" (by erf) or "silu"; add: [rows, out] of dtype, a residual.  With pre=True (out, x @ weight + bias),
    the second for linear_grad."""
    return _forward("linear", x, None, weight, bias, act, add, pre, dtype)


def grouped_linear(xs, offsets, weight, bias=None, act=None, add=None, pre=False, dtype=None):
    """linear with every expert's own weights, on rows sorted by expert: rows offsets[e] .. offsets[e + 1] of xs take weight[e] and
    bias[e]; rows behind offsets[-1] are zero (and not read).

    xs, offsets: as dispatch gives them; weight: [experts, in, out]; bias: [experts, out]; the rest as in linear."""
    if offsets is None:
        _refuse("offsets is None")
    return _forward("grouped_linear", xs, offsets, weight, bias, act, add, pre, dtype)


def _backward(name, dout, x, offsets, weight, pre, act, dtype, for_x, for_weight, for_bias):
    dtype_code, dstride = _rows(dout, "dout")
    dev = dout.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return _backward(name, dout, x, offsets, weight, pre, act, dtype, for_x, for_weight, for_bias)
    if _asks(dout, x, weight, pre):
        _unrecorded(name, 4)
    xtype, xstride = _rows(x, "x", dev)
    sets = offsets is not None
    op = _offsets(offsets, weight, x) if sets else 0
    experts, width, cols, transposed, wstride, estride = _weight(weight, x, sets)
    rows = x.shape[0]
    if dout.shape != (rows, cols):
        _refuse("dout: %s, not %s", (rows, cols), tuple(dout.shape))
    act = _act(act)
    pp, pstride = 0, cols
    if act != SPDNN_ACT_NONE:
        if pre is None:
            _refuse("pre is None, with an activation")
        ptype, pstride = _rows(pre, "pre", dev, (rows, cols))
        if ptype != dtype_code:
            _refuse("pre: %s, not %s", dout.dtype, pre.dtype)
        pp = pre.data_ptr()
    dtype = x.dtype if dtype is None else dtype
    gtype = _type(dtype, "dtype")
    need = _work_bytes("spdnn_linear_grad_bytes", rows, width, cols, sets, experts, xtype, dtype_code, act, transposed)
    dx = torch.empty((rows, width), dtype=x.dtype, device=dev) if for_x else None
    dweight = dbias = None
    first = (experts,) if sets else ()
    if for_weight:  # stored as weight is
        dweight = weight.new_empty(first + ((cols, width) if transposed else (width, cols)), dtype=dtype)
    if for_bias:
        dbias = weight.new_empty(first + (cols,), dtype=dtype)
    work = x.new_empty(need, dtype=torch.uint8) if need else None
    _check(lib().spdnn_linear_grad(dout.data_ptr(), dtype_code, dstride, pp, pstride, act, x.data_ptr(), xtype, rows, width, xstride, op, experts,
                                   weight.data_ptr(), transposed, wstride, estride, cols, dx.data_ptr() if for_x else 0, width,
                                   dweight.data_ptr() if for_weight else 0, width if transposed else cols, width * cols,
                                   dbias.data_ptr() if for_bias else 0, gtype, work.data_ptr() if need else 0, need, _stream(dev.index)))
    return dx, dweight.transpose(-1, -2) if transposed and for_weight else dweight, dbias


def linear_grad(dout, x, weight, pre=None, act=None, dtype=None, for_x=True, for_weight=True, for_bias=True):
    """(dx, dweight, dbias): gradients of linear (that of add is dout).

    dout: [rows, out] of x's type or float32; act as it was there, pre as linear gave it (of dout's type), needed with an act.  dx is
    of x's type; dweight and dbias are of dtype (x's, or float32), dweight is stored as weight is.  dout times the activation's slope
    is rounded to x's type for dx and dweight (in float16 what lies beyond 65504 is infinite there); dbias sums it in 32 bits.
    What for_x, for_weight and for_bias leave out is None."""
    return _backward("linear_grad", dout, x, None, weight, pre, act, dtype, for_x, for_weight, for_bias)


def grouped_linear_grad(dout, xs, offsets, weight, pre=None, act=None, dtype=None, for_x=True, for_weight=True, for_bias=True):
    """(dxs, dweight [experts, in, out], dbias [experts, out]): gradients of grouped_linear; dxs is zero in rows of no expert, dweight and
    dbias for experts without rows.  The rest as in linear_grad."""
    if offsets is None:
        _refuse("offsets is None")
    return _backward("grouped_linear_grad", dout, xs, offsets, weight, pre, act, dtype, for_x, for_weight, for_bias)


def layer_norm(x, weight=None, bias=None, eps=1e-5, stats=False, dtype=None):
    """(x - mean) * rstd * weight + bias over every row, rstd = 1 / sqrt(variance + eps): [rows, width] of dtype (x's, or float32).

    weight, bias: [width], both of x's type or both float32; ones and zeros if None.  With stats=True (out, float32 [rows, 2] of mean
    and rstd), the second for layer_norm_grad."""
    xtype, xstride = _rows(x, "x")
    rows, width = x.shape
    dev = x.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return layer_norm(x, weight, bias, eps, stats, dtype)
    if _asks(x, weight, bias):
        _unrecorded("layer_norm")
    otype = xtype if dtype is None else _type(dtype, "dtype")
    wp, wtype = _vector(weight, "weight", x, (width,))
    bp, btype = _vector(bias, "bias", x, (width,))
    if weight is not None and bias is not None and wtype != btype:
        _refuse("bias: %s, not %s", weight.dtype, bias.dtype)
    out = x.new_empty((rows, width), dtype=dtype)
    kept = torch.empty((rows, 2), dtype=torch.float32, device=dev) if stats else None
    _check(lib().spdnn_layer_norm(x.data_ptr(), xtype, rows, width, xstride, wp, bp, wtype if wp else btype, eps, out.data_ptr(), otype, width,
                                  kept.data_ptr() if stats else 0, _stream(dev.index)))
    return (out, kept) if stats else out


def layer_norm_grad(dout, x, stats, weight=None, add=None, dtype=None, for_weight=True, for_bias=True):
    """(dx, dweight, dbias): gradients of layer_norm, with stats as it gave them.

    dout: of x's type; add: a gradient that x has from elsewhere (in a residual block), added to dx.  dweight and dbias are of dtype
    (weight's, or float32 if that is None); what for_weight and for_bias leave out is None."""
    xtype, xstride = _rows(x, "x")
    rows, width = x.shape
    dev = x.device
    if dev.index != _current():
        with torch.cuda.device(dev):
            return layer_norm_grad(dout, x, stats, weight, add, dtype, for_weight, for_bias)
    if _asks(dout, x, weight, add):
        _unrecorded("layer_norm_grad")
    dcode, dstride = _rows(dout, "dout", dev, (rows, width))
    if dcode != xtype:
        _refuse("dout: %s, not %s", x.dtype, dout.dtype)
    if stats is None:
        _refuse("stats is None")
    sp = _array(stats, "stats", _F32, dev, (rows, 2))
    wp, wtype = _vector(weight, "weight", x, (width,))
    ap, astride = 0, width
    if add is not None:
        atype, astride = _rows(add, "add", dev, (rows, width))
        if atype != xtype:
            _refuse("add: %s, not %s", x.dtype, add.dtype)
        ap = add.data_ptr()
    dtype = (torch.float32 if weight is None else weight.dtype) if dtype is None else dtype
    gtype = _type(dtype, "dtype")
    need = _work_bytes("spdnn_layer_norm_grad_bytes", rows, width) if for_weight or for_bias else 0
    dx = torch.empty((rows, width), dtype=x.dtype, device=dev)
    dweight = torch.empty(width, dtype=dtype, device=dev) if for_weight else None
    dbias = torch.empty(width, dtype=dtype, device=dev) if for_bias else None
    work = x.new_empty(need, dtype=torch.uint8) if need else None
    _check(lib().spdnn_layer_norm_grad(dout.data_ptr(), xtype, dstride, x.data_ptr(), rows, width, xstride, sp, wp, wtype, ap, astride, dx.data_ptr(),
                                       width, dweight.data_ptr() if for_weight else 0, dbias.data_ptr() if for_bias else 0, gtype,
                                       work.data_ptr() if need else 0, need, _stream(dev.index)))
    return dx, dweight, dbias

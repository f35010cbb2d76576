"""Row operators: what the C entry points refuse before any HIP call, and sizes of their work memory."""
import ctypes

import numpy as np
import pytest

import paper_2007_14152_amd as sp

P = 256 * 4096  # an aligned address that is never dereferenced


def call(name, **changes):
    """The entry point with arguments that are fine but for the changes."""
    args = {
        "spdnn_embed": dict(table=P, table_type=0, vocab=10, width=8, table_stride=8, ids=P, ids_type=0, n=3, scale=1.0, out=P,
                            out_type=0, out_stride=8, stream=None),
        "spdnn_embed_grad": dict(dout=P, dout_type=0, dout_stride=8, ids=P, ids_type=0, n=3, vocab=10, width=8, scale=1.0, accumulate=0,
                                 dtable=P, dtable_type=0, dtable_stride=8, work=P, work_bytes=1 << 40, stream=None),
        "spdnn_route": dict(logits=P, type=0, stride=8, rows=3, experts=8, k=2, bias=None, keep=None, score=0, normalise=1, scale=1.0,
                            chosen=P, weight=P, stream=None),
        "spdnn_route_grad": dict(dweight=P, logits=P, type=0, stride=8, chosen=P, rows=3, experts=8, k=2, bias=None, score=0, normalise=1,
                                 scale=1.0, dlogits=P, dstride=8, stream=None),
        "spdnn_dispatch": dict(chosen=P, rows=3, k=2, experts=8, x=P, type=0, width=8, x_stride=8, xs=P, xs_stride=8, offsets=P, place=P,
                               work=P, work_bytes=1 << 40, stream=None),
        "spdnn_combine": dict(ys=P, type=0, width=8, ys_stride=8, place=P, weight=P, rows=3, k=2, add=None, add_stride=0, out=P,
                              out_stride=8, stream=None),
        "spdnn_combine_grad": dict(dout=P, type=0, width=8, dout_stride=8, ys=P, ys_stride=8, place=P, weight=P, count=P, rows=3, k=2,
                                   dys=P, dys_stride=8, dweight=P, stream=None),
    }[name]
    assert set(changes) <= set(args)
    args.update(changes)
    return getattr(sp.lib(), name)(*args.values())


REFUSED = [
    ("spdnn_embed", [dict(table=None), dict(out=None), dict(ids=None), dict(vocab=0), dict(width=0), dict(n=-1), dict(table_type=3),
                     dict(out_type=-1), dict(ids_type=2), dict(out_stride=7), dict(table_stride=-1), dict(table=P + 2), dict(ids=P + 2),
                     dict(ids=P + 4, ids_type=1), dict(out=P + 1, out_type=1), dict(table_stride=1 << 62)]),
    ("spdnn_embed_grad", [dict(dout=None), dict(dtable=None), dict(ids=None), dict(vocab=0), dict(width=-3), dict(n=-1), dict(dout_type=7),
                          dict(dtable_type=4), dict(ids_type=-1), dict(dtable_stride=7), dict(dtable=P + 2), dict(work=P + 128)]),
    ("spdnn_route", [dict(logits=None), dict(chosen=None), dict(weight=None), dict(rows=-1), dict(k=0), dict(k=9), dict(experts=0),
                     dict(experts=1025, stride=1025), dict(experts=100, stride=100, k=17), dict(score=2), dict(type=9), dict(stride=-8),
                     dict(bias=P + 2), dict(chosen=P + 2), dict(weight=P + 1)]),
    ("spdnn_route_grad", [dict(dweight=None), dict(logits=None), dict(chosen=None), dict(dlogits=None), dict(dstride=7), dict(k=9),
                          dict(score=-1), dict(dlogits=P + 2), dict(dweight=P + 2)]),
    ("spdnn_dispatch", [dict(chosen=None), dict(x=None), dict(xs=None), dict(offsets=None), dict(place=None), dict(rows=-1), dict(k=0),
                        dict(k=17), dict(experts=0), dict(experts=1025), dict(width=0), dict(xs_stride=7), dict(rows=1 << 30), dict(type=5),
                        dict(work=P + 4), dict(xs=P + 2), dict(place=P + 2), dict(offsets=P + 1)]),
    ("spdnn_combine", [dict(ys=None), dict(place=None), dict(out=None), dict(k=0), dict(rows=-2), dict(width=0), dict(out_stride=4),
                       dict(ys_stride=-1), dict(add=P + 2), dict(weight=P + 2), dict(rows=1 << 30, k=2)]),
    ("spdnn_combine_grad", [dict(dout=None), dict(ys=None), dict(place=None), dict(weight=None), dict(count=None), dict(dys=None),
                            dict(dweight=None), dict(dys_stride=7), dict(k=17), dict(width=0), dict(type=-1), dict(dweight=P + 2)]),
]


W = (1 << 30) + 1  # a row too long
REFUSED += [("spdnn_embed", [dict(width=W, table_stride=W, out_stride=W)]), ("spdnn_embed_grad", [dict(width=W, dout_stride=W, dtable_stride=W)]),
            ("spdnn_dispatch", [dict(width=W, x_stride=W, xs_stride=W)]), ("spdnn_combine", [dict(width=W, ys_stride=W, out_stride=W)]),
            ("spdnn_combine_grad", [dict(width=W, dout_stride=W, ys_stride=W, dys_stride=W)])]


@pytest.mark.parametrize("name,changes", [(n, c) for n, cs in REFUSED for c in cs], ids=lambda v: str(v))
def test_refused_before_touching_the_gpu(name, changes):
    assert call(name, **changes) == sp.SPDNN_EINVAL
    assert sp.spdnn_last_error() != ""


def test_work_memory():
    size = ctypes.c_size_t()
    for name, args in [("spdnn_embed_grad_bytes", (50000, 1024, 1)), ("spdnn_embed_grad_bytes", (1, 1, 0)),
                       ("spdnn_embed_grad_bytes", (2 ** 31 - 1, 1 << 30, 2 ** 31 - 1)), ("spdnn_dispatch_bytes", (0, 1, 1)),
                       ("spdnn_dispatch_bytes", (1 << 26, 16, 1024))]:
        assert getattr(sp.lib(), name)(*args, ctypes.byref(size)) == sp.SPDNN_OK
        assert getattr(sp.lib(), name)(*args, None) == sp.SPDNN_EINVAL
    for name, bad in [("spdnn_embed_grad_bytes", [(0, 1, 1), (1, 0, 1), (1, 1, -1)]),
                      ("spdnn_dispatch_bytes", [(-1, 1, 1), (1, 0, 1), (1, 17, 20), (1, 1, 0), (1, 1, 1025), (1 << 30, 2, 4)])]:
        for args in bad:
            assert getattr(sp.lib(), name)(*args, ctypes.byref(size)) == sp.SPDNN_EINVAL, args


@pytest.mark.parametrize("name,sizes", [("spdnn_dispatch", dict(rows=100000, k=8, experts=256)),
                                        ("spdnn_embed_grad", dict(n=100000, vocab=50000, width=64, dout_stride=64, dtable_stride=64))])
def test_work_memory_that_is_too_small(name, sizes):
    size = ctypes.c_size_t()
    if name == "spdnn_dispatch":
        sp.lib().spdnn_dispatch_bytes(sizes["rows"], sizes["k"], sizes["experts"], ctypes.byref(size))
    else:
        sp.lib().spdnn_embed_grad_bytes(sizes["vocab"], sizes["width"], sizes["n"], ctypes.byref(size))
    if size.value:
        assert call(name, work_bytes=size.value - 1, **sizes) == sp.SPDNN_ESIZE
        assert call(name, work_bytes=size.value, work=None, **sizes) == sp.SPDNN_EINVAL


def test_reference_against_dense_formulas():
    """The 64-bit reference itself, against torch's automatic gradients of the dense formulas on the CPU."""
    import torch

    import rows_ref as ref
    g = torch.Generator().manual_seed(1)
    rows, experts, k = 9, 6, 3
    for score, normalise in [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)]:
        l = torch.randn(rows, experts, generator=g, dtype=torch.float64, requires_grad=True)
        chosen, is_open = ref.choose(l.detach().numpy().astype(np.float32), k)
        p = torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)
        w = p.gather(1, torch.from_numpy(chosen).long())
        if normalise:
            w = w / w.sum(1, keepdim=True)
        w = 1.5 * w
        dw = torch.randn(rows, k, generator=g, dtype=torch.float64)
        (w * dw).sum().backward()
        assert np.allclose(ref.weights(l.detach().numpy(), is_open, chosen, score, normalise, 1.5), w.detach().numpy(), rtol=1e-12)
        d, _ = ref.route_grad(dw.numpy(), l.detach().numpy(), is_open, chosen, score, normalise, 1.5)
        assert np.allclose(d, l.grad.numpy(), rtol=1e-10, atol=1e-13)
    ids = torch.tensor([3, 1, -1, 3, 0])
    dout = torch.randn(5, 4, generator=g, dtype=torch.float64)
    table = torch.zeros(4, 4, dtype=torch.float64, requires_grad=True)
    (2.0 * table[ids.clamp(min=0)] * (ids >= 0)[:, None] * dout).sum().backward()
    assert np.allclose(ref.embed_grad(dout.numpy(), ids.numpy(), 4, 2.0)[0], table.grad.numpy())
    place, offsets = ref.sort_pairs(np.array([[2, 0], [-1, 2], [0, 1]], dtype=np.int32), 3)
    assert place.tolist() == [[3, 0], [-1, 4], [1, 2]] and offsets.tolist() == [0, 2, 3, 5]

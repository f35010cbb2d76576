"""Dense products and layer norm: what the C entry points refuse before any HIP call, sizes of their work memory, and what the binding
refuses before the library sees it."""
import ctypes

import pytest
import torch

import paper_2007_14152_amd as sp
from paper_2007_14152_amd import dense, rows

P = 256 * 4096  # an aligned address that is never dereferenced


def call(name, **changes):
    """The entry point with arguments that are fine but for the changes."""
    args = {
        "spdnn_linear": dict(x=P, type=0, rows=3, width=8, x_stride=8, offsets=P, experts=2, weight=P, transposed=0, weight_stride=16,
                             expert_stride=128, cols=16, bias=P, bias_type=0, act=1, add=P, add_stride=16, out=P, out_type=0, out_stride=16,
                             pre=P, pre_stride=16, work=P, work_bytes=1 << 40, stream=None),
        "spdnn_linear_grad": dict(dout=P, dout_type=0, dout_stride=16, pre=P, pre_stride=16, act=1, x=P, type=0, rows=3, width=8, x_stride=8,
                                  offsets=P, experts=2, weight=P, transposed=0, weight_stride=16, expert_stride=128, cols=16, dx=P, dx_stride=8,
                                  dweight=P, dweight_stride=16, dexpert_stride=128, dbias=P, grad_type=0, work=P, work_bytes=1 << 40, stream=None),
        "spdnn_layer_norm": dict(x=P, type=0, rows=3, width=8, x_stride=8, weight=P, bias=P, param_type=0, eps=1e-5, out=P, out_type=0,
                                 out_stride=8, stats=P, stream=None),
        "spdnn_layer_norm_grad": dict(dout=P, type=0, dout_stride=8, x=P, rows=3, width=8, x_stride=8, stats=P, weight=P, param_type=0, add=P,
                                      add_stride=8, dx=P, dx_stride=8, dweight=P, dbias=P, grad_type=0, work=P, work_bytes=1 << 40, stream=None),
    }[name]
    assert set(changes) <= set(args)
    args.update(changes)
    return getattr(sp.lib(), name)(*args.values())


W = (1 << 30) + 1  # too long
REFUSED = [
    ("spdnn_linear", [dict(x=None), dict(weight=None), dict(out=None), dict(offsets=None), dict(rows=-1), dict(width=0), dict(cols=0), dict(experts=0),
                      dict(experts=1025), dict(type=3), dict(type=-1), dict(out_type=1), dict(type=1, bias_type=2, out_type=1), dict(bias_type=1), dict(act=5),
                      dict(act=-1), dict(x_stride=-1), dict(weight_stride=-1), dict(expert_stride=-1), dict(out_stride=15), dict(pre_stride=15),
                      dict(add_stride=-2), dict(x=P + 2), dict(weight=P + 2), dict(bias=P + 2), dict(add=P + 1), dict(out=P + 2), dict(pre=P + 2),
                      dict(offsets=P + 2), dict(width=W, x_stride=W), dict(cols=W, out_stride=W, pre_stride=W), dict(expert_stride=1 << 60),
                      dict(x_stride=1 << 62), dict(rows=2 ** 31 - 1, cols=1 << 30, out_stride=1 << 30, pre_stride=1 << 30)]),
    ("spdnn_linear_grad", [dict(dout=None), dict(pre=None), dict(x=None), dict(weight=None), dict(offsets=None), dict(rows=-1), dict(width=0),
                           dict(cols=-4), dict(experts=0), dict(type=7), dict(dout_type=2), dict(act=9), dict(grad_type=1), dict(dx_stride=7),
                           dict(dweight_stride=15), dict(dexpert_stride=127), dict(transposed=1, dweight_stride=7, dexpert_stride=512), dict(dx=P + 2),
                           dict(dweight=P + 2), dict(dbias=P + 2), dict(dout=P + 2), dict(pre=P + 2), dict(x=P + 1), dict(work=P + 128),
                           dict(offsets=P + 1), dict(width=W, x_stride=W, dx_stride=W)]),
    ("spdnn_layer_norm", [dict(x=None), dict(out=None), dict(rows=-1), dict(width=0), dict(type=5), dict(out_type=1), dict(param_type=1), dict(eps=-1.0),
                          dict(eps=float("nan")), dict(out_stride=7), dict(x_stride=-1), dict(x=P + 2), dict(weight=P + 2), dict(bias=P + 2),
                          dict(stats=P + 4), dict(width=W, x_stride=W, out_stride=W)]),
    ("spdnn_layer_norm_grad", [dict(dout=None), dict(x=None), dict(stats=None), dict(dx=None), dict(rows=-1), dict(width=0), dict(type=5),
                               dict(param_type=2), dict(grad_type=1), dict(dx_stride=7), dict(dx=P + 2), dict(dweight=P + 2), dict(dbias=P + 2),
                               dict(stats=P + 4), dict(add=P + 2), dict(add_stride=-1), dict(work=P + 64), dict(work=None)]),
]


@pytest.mark.parametrize("name,changes", [(n, c) for n, cs in REFUSED for c in cs], ids=lambda v: str(v))
def test_refused_before_touching_the_gpu(name, changes):
    assert call(name, **changes) == sp.SPDNN_EINVAL
    assert sp.spdnn_last_error() != ""


def test_nothing_to_do():
    """Without rows nothing is launched that needs them."""
    assert call("spdnn_linear", rows=0, x=None, out=None, pre=None, add=None) == sp.SPDNN_OK
    assert call("spdnn_layer_norm", rows=0, x=None, out=None) == sp.SPDNN_OK


def test_work_memory():
    size = ctypes.c_size_t()
    L = sp.lib()

    def ask(name, *args):
        assert getattr(L, name)(*args, ctypes.byref(size)) == sp.SPDNN_OK, sp.spdnn_last_error()
        assert getattr(L, name)(*args, None) == sp.SPDNN_EINVAL
        assert size.value % 256 == 0
        return size.value

    for args in [(0, 1, 1, 0, 1, 0), (1, 4096, 16384, 0, 1, 1), (24000, 4096, 4096, 1, 64, 2), (1 << 20, 4096, 16384, 0, 1, 1)]:
        ask("spdnn_linear_bytes", *args)
    assert ask("spdnn_linear_grad_bytes", 1000, 64, 40, 0, 1, 1, 1, 3, 0) >= 1000 * 40 * 2  # rows of d
    assert ask("spdnn_linear_grad_bytes", 1000, 64, 40, 0, 1, 1, 0, 0, 0) >= 1000 * 40 * 2
    ask("spdnn_linear_grad_bytes", 48000, 4096, 4096, 1, 64, 1, 1, 0, 1)
    assert ask("spdnn_layer_norm_grad_bytes", 3, 100) >= 3 * 2 * 100 * 4
    ask("spdnn_layer_norm_grad_bytes", 0, 1)
    ask("spdnn_layer_norm_grad_bytes", 2 ** 31 - 1, 1 << 30)
    need = ask("spdnn_layer_norm_grad_bytes", 3, 8)
    assert call("spdnn_layer_norm_grad", work_bytes=need - 1) == sp.SPDNN_ESIZE
    assert call("spdnn_linear_grad", work_bytes=0) == sp.SPDNN_ESIZE
    for bad in [(-1, 8, 8, 0, 1, 0), (1, 0, 8, 0, 1, 0), (1, 8, 0, 0, 1, 0), (1, 8, 8, 0, 0, 0), (1, 8, 8, 0, 1025, 0), (1, 8, 8, 0, 1, 3)]:
        assert L.spdnn_linear_bytes(*bad, ctypes.byref(size)) == sp.SPDNN_EINVAL
        assert L.spdnn_linear_grad_bytes(*bad, 0, 0, 0, ctypes.byref(size)) == sp.SPDNN_EINVAL
    # A launch takes less than 2^32 threads: more tiles are refused, long and thin outputs within it are not.
    for big in [(2 ** 31 - 1, 1, 1, 0, 1, 1), (1 << 20, 8, 1 << 24, 0, 1, 1), (1000, 8, 1 << 30, 0, 1, 0)]:
        assert L.spdnn_linear_bytes(*big, ctypes.byref(size)) == sp.SPDNN_EINVAL and "tiles" in sp.spdnn_last_error()
    assert L.spdnn_linear_grad_bytes(8, 1 << 24, 1 << 14, 1, 256, 1, 1, 0, 0, ctypes.byref(size)) == sp.SPDNN_EINVAL
    for type in (0, 1, 2):
        ask("spdnn_linear_bytes", (1 << 30) - 1, 64, 64, 0, 1, type)
        ask("spdnn_linear_bytes", (1 << 29) - 1, 4096, 1, 1, 1024, type)
        ask("spdnn_linear_grad_bytes", 100, (1 << 29) - 1, 1, 0, 1, type, type, 0, 1)  # (dx: 2^22 tiles of 128 x 128; 1000 rows are 2^25)


def test_work_memory_of_long_rows():
    """Rows that registers do not hold in any type leave 16 parts, whatever their number: no more memory than that is asked for."""
    size = ctypes.c_size_t()
    for rows, width in [(600, 1 << 20), (4096, 65536), (600, 40000), (9, 32769), (2 ** 31 - 1, 1 << 30)]:
        assert sp.lib().spdnn_layer_norm_grad_bytes(rows, width, ctypes.byref(size)) == sp.SPDNN_OK
        assert 0 <= size.value - min(rows, 16) * 2 * width * 4 < 256
    for rows, width in [(600, 16385), (4096, 32768), (9, 32768)]:
        assert sp.lib().spdnn_layer_norm_grad_bytes(rows, width, ctypes.byref(size)) == sp.SPDNN_OK
        assert 0 <= size.value - min(rows, 512) * 2 * width * 4 < 256


class Shape:
    """A tensor without memory that says that it lies on the GPU."""

    def __init__(self, *shape, dtype=torch.float32, like=None):
        self.t = torch.empty(shape, dtype=dtype, device="meta") if like is None else like
        self.is_cuda, self.device = True, torch.device("cuda:0")

    def __getattr__(self, name):
        return getattr(self.t, name)

    def transpose(self, *dims):
        return Shape(like=self.t.transpose(*dims))


@pytest.fixture
def no_gpu(monkeypatch):
    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):  # asked for sizes only
                return getattr(sp.lib(), name)
            raise AssertionError("%s would have been called" % name)

    for module in (rows, dense):
        monkeypatch.setattr(module, "_current", lambda: 0)
        monkeypatch.setattr(module, "lib", Library)
    rows._work_bytes.cache_clear()


S = Shape
BIG = 2 ** 32 + 5
BF = torch.bfloat16


def off(n):
    return S(n, dtype=torch.int32)


BINDING = [
    lambda: dense.linear(S(3, 8), S(8)),
    lambda: dense.linear(S(3, 8), S(2, 8, 4)),
    lambda: dense.linear(S(3, 8), S(9, 4)),
    lambda: dense.linear(S(3, 8), S(8, 4, dtype=BF)),
    lambda: dense.linear(S(3, 8, dtype=torch.float64), S(8, 4, dtype=torch.float64)),
    lambda: dense.linear(S(2, 3, 8), S(8, 4)),
    lambda: dense.linear(S(3, 8), S(8, 4), act="tanh"),
    lambda: dense.linear(S(3, 8), S(8, 4), act=1),
    lambda: dense.linear(S(3, 8), S(8, 4), bias=S(5)),
    lambda: dense.linear(S(3, 8), S(8, 4), bias=S(4, dtype=BF)),
    lambda: dense.linear(S(3, 8), S(8, 4), add=S(3, 5)),
    lambda: dense.linear(S(3, 8, dtype=BF), S(8, 4, dtype=BF), add=S(3, 4), dtype=BF),
    lambda: dense.linear(S(3, 8, dtype=BF), S(8, 4, dtype=BF), dtype=torch.int32),
    lambda: dense.linear(S(3, 8), Shape(like=torch.empty(8, 4, 2, device="meta")[:, :, 0])),
    lambda: dense.linear(S(3, BIG), S(BIG, 4)),
    lambda: dense.linear(S(BIG, 8), S(8, 4)),
    lambda: dense.linear(S(3, 8), S(8, BIG)),
    lambda: dense.grouped_linear(S(3, 8), None, S(2, 8, 4)),
    lambda: dense.grouped_linear(S(3, 8), off(2), S(2, 8, 4)),
    lambda: dense.grouped_linear(S(3, 8), S(3), S(2, 8, 4)),
    lambda: dense.grouped_linear(S(3, 8), off(3), S(8, 4)),
    lambda: dense.grouped_linear(S(3, 8), off(3), S(2, 8, 4), bias=S(4)),
    lambda: dense.grouped_linear(S(3, 8), off(BIG + 1), S(BIG, 8, 4)),
    lambda: dense.linear_grad(S(3, 5), S(3, 8), S(8, 4)),
    lambda: dense.linear_grad(S(4, 4), S(3, 8), S(8, 4)),
    lambda: dense.linear_grad(S(3, 4), S(3, 8), S(8, 4), act="gelu"),
    lambda: dense.linear_grad(S(3, 4), S(3, 8), S(8, 4), act="gelu", pre=S(3, 4, dtype=BF)),
    lambda: dense.linear_grad(S(3, 4), S(3, 8), S(8, 4), act="gelu", pre=S(3, 5)),
    lambda: dense.linear_grad(S(3, 4, dtype=BF), S(3, 8), S(8, 4)),
    lambda: dense.linear_grad(S(3, 4), S(3, 8), S(8, 4), dtype=torch.float64),
    lambda: dense.grouped_linear_grad(S(3, 4), S(3, 8), None, S(2, 8, 4)),
    lambda: dense.grouped_linear_grad(S(3, 4), S(3, 8), off(4), S(2, 8, 4)),
    lambda: dense.layer_norm(S(8)),
    lambda: dense.layer_norm(S(3, 8), S(7)),
    lambda: dense.layer_norm(S(3, 8, dtype=BF), S(8), S(8, dtype=BF)),
    lambda: dense.layer_norm(S(3, 8), dtype=torch.float64),
    lambda: dense.layer_norm(S(3, BIG)),
    lambda: dense.layer_norm_grad(S(3, 8), S(3, 8), None),
    lambda: dense.layer_norm_grad(S(3, 8), S(3, 8), S(3, 3)),
    lambda: dense.layer_norm_grad(S(3, 8, dtype=BF), S(3, 8), S(3, 2)),
    lambda: dense.layer_norm_grad(S(3, 7), S(3, 8), S(3, 2)),
    lambda: dense.layer_norm_grad(S(3, 8), S(3, 8), S(3, 2), add=S(2, 8)),
    lambda: dense.layer_norm_grad(S(3, 8), S(3, 8), S(3, 2), dtype=torch.float64),
]


@pytest.mark.parametrize("i", range(len(BINDING)))
def test_the_binding_refuses(no_gpu, i):
    with pytest.raises(sp.SpdnnError):
        BINDING[i]()


def test_how_weights_are_stored():
    def stored(t, x):
        return dense._weight(t, x, t.dim() == 3)[3:]

    x = S(3, 8)
    assert stored(S(8, 4), x) == (False, 4, 0)
    assert stored(S(4, 8).transpose(0, 1), x) == (True, 8, 0)
    assert stored(S(2, 8, 4), x) == (False, 4, 32)
    assert stored(S(2, 4, 8).transpose(1, 2), x) == (True, 8, 32)
    assert stored(Shape(like=torch.empty(8, 100, device="meta")[:, 3:9]), x) == (False, 100, 0)
    assert stored(S(8, 1), x)[0] is True  # a column: its rows are adjacent
    assert stored(S(1, 4), S(3, 1))[0] in (False, True)
    assert stored(Shape(like=torch.empty(8, 4, device="meta").expand(5, 8, 4)), x) == (False, 4, 0)


def test_a_weight_of_one_row():
    """One row has adjacent rows, whatever lies between its columns."""
    x = S(3, 1)
    one = Shape(like=torch.empty(6, 4, 5, device="meta")[:1, :, 2])
    assert one.stride() == (20, 5)
    assert dense._weight(one, x, False) == (1, 1, 4, True, 5, 0)
    many = Shape(like=torch.empty(2, 6, 4, 5, device="meta")[:, :1, :, 2])
    assert dense._weight(many, x, True) == (2, 1, 4, True, 5, 120)
    assert dense._weight(S(1, 4), x, False) == (1, 1, 4, False, 4, 0)
    assert dense._weight(Shape(like=torch.empty(1, 1, device="meta").expand(1, 4)), x, False)[3:5] == (True, 0)  # one number for all columns

"""Row operators: sizes that 32 bits do not hold are refused before the library sees them (the binding would pass on what is
left of them).  Tensors without memory stand for those of the GPU."""
import pytest
import torch

import paper_2007_14152_amd as sp
from paper_2007_14152_amd import rows

BIG = 2 ** 32 + 5  # 5 in 32 bits


class Shape:
    """A tensor without memory that says that it lies on the GPU."""

    def __init__(self, *shape, dtype=torch.float32):
        self.t = torch.empty(shape, dtype=dtype, device="meta")
        self.is_cuda, self.device = True, torch.device("cuda:0")

    def __getattr__(self, name):
        return getattr(self.t, name)

    def contiguous(self):
        return self


@pytest.fixture
def no_gpu(monkeypatch):
    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):  # asked for sizes only
                return getattr(sp.lib(), name)
            raise AssertionError("%s would have been called" % name)

    monkeypatch.setattr(rows, "_current", lambda: 0)
    monkeypatch.setattr(rows, "lib", Library)
    rows._work_bytes.cache_clear()


def ids(*shape):
    return Shape(*shape, dtype=torch.int32)


CALLS = [
    lambda: rows.embed(Shape(BIG, 8), ids(3)),
    lambda: rows.embed(Shape(9, BIG), ids(3)),
    lambda: rows.embed(Shape(9, 8), ids(BIG)),
    lambda: rows.embed(Shape(9, 8), ids(2 ** 16, 2 ** 16)),
    lambda: rows.embed_grad(Shape(BIG, 8), ids(BIG), 9),
    lambda: rows.embed_grad(Shape(3, BIG), ids(3), 9),
    lambda: rows.embed_grad(Shape(3, 8), ids(3), BIG),
    lambda: rows.embed_grad(Shape(3, 8), ids(3), 5 - 2 ** 32),
    lambda: rows.embed_grad(Shape(3, 8), ids(3), BIG, out=Shape(BIG, 8)),
    lambda: rows.route(Shape(BIG, 8), 2),
    lambda: rows.route(Shape(3, BIG), 2),
    lambda: rows.route(Shape(3, 8), BIG),
    lambda: rows.route(Shape(3, 8), 5 - 2 ** 32),
    lambda: rows.route_grad(Shape(BIG, 2), Shape(BIG, 8), ids(BIG, 2)),
    lambda: rows.route_grad(Shape(0, BIG), Shape(0, 8), ids(0, BIG)),
    lambda: rows.dispatch(Shape(BIG, 8), ids(BIG, 2), 4),
    lambda: rows.dispatch(Shape(3, BIG), ids(3, 2), 4),
    lambda: rows.dispatch(Shape(0, 8), ids(0, BIG), 4),
    lambda: rows.dispatch(Shape(3, 8), ids(3, 2), BIG),
    lambda: rows.combine(Shape(2 * BIG, 8), ids(BIG, 2)),
    lambda: rows.combine(Shape(6, BIG), ids(3, 2)),
    lambda: rows.combine(Shape(0, 8), ids(0, BIG)),
    lambda: rows.dispatch_grad(Shape(0, 8), ids(0, BIG)),
    lambda: rows.combine_grad(Shape(BIG, 8), Shape(2 * BIG, 8), ids(BIG, 2), Shape(BIG, 2), ids(5)),
    lambda: rows.combine_grad(Shape(0, 8), Shape(0, 8), ids(0, BIG), Shape(0, BIG), ids(5)),
]


@pytest.mark.parametrize("number", range(len(CALLS)))
def test_sizes_beyond_32_bits_are_refused(no_gpu, number):
    with pytest.raises(sp.SpdnnError) as e:
        CALLS[number]()
    assert e.value.code == sp.SPDNN_EINVAL


def test_work_memory_of_sizes_beyond_32_bits(no_gpu):
    for name in ("spdnn_embed_grad_bytes", "spdnn_dispatch_bytes"):
        assert rows._work_bytes(name, 3000, 8, 8) >= 0
        for sizes in ((2 ** 32 + 3000, 8, 8), (3000, 2 ** 32 + 8, 8), (3000, 8, 2 ** 32 + 8), (3000, 8, 8 - 2 ** 32), (2 ** 31, 8, 8)):
            with pytest.raises(sp.SpdnnError):
                rows._work_bytes(name, *sizes)

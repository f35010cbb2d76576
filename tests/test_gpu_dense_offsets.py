"""Offsets that do not ascend within 0 .. rows: the rows are not specified, nothing outside the arrays is written.  Over the types, both
storage orders, and sizes that come to large tiles and to k in parts."""
import ctypes

import pytest
import torch

import dense_plans as plans

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ROOM = 1 << 15  # bytes on either side


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


class Guarded:
    """Memory with a known pattern around it."""

    def __init__(self, count, size):
        self.bytes = count * size
        self.t = torch.full((self.bytes + 2 * ROOM,), 0x55, dtype=torch.uint8, device=DEV)
        self.p = self.t.data_ptr() + ROOM

    def whole(self):
        return bool((self.t[:ROOM] == 0x55).all()) and bool((self.t[ROOM + self.bytes:] == 0x55).all())


def wrong(rows, n):
    """Some ways, for n experts."""
    top, low = 2 ** 31 - 1, -2 ** 31
    return [[0, rows] * n, [rows, 0] * n, [-5, rows + 900, 7] * n, [top] * (n + 1), [low] * (n + 1), [low, top] * n, list(range(rows, rows - n - 1, -1)), [rows // 2] * (n + 1),
            [rows // 3] + [rows] * n]


SIZES = [(n, l, d, k, c) for n, l, d, k, c in plans.GROUPED_16 + plans.GROUPED_32[2:] if k * c * sum(l) < 5e9] + [("few", l, d, k, c) for l, d, k, c in plans.FEW_GROUPED]


@pytest.mark.parametrize("transposed", [0, 1])
@pytest.mark.parametrize("dtype,act", [(torch.float32, 0), (torch.float32, 3), (torch.bfloat16, 0), (torch.float16, 3)])
@pytest.mark.parametrize("loads,dropped,width,cols", [s[1:] for s in SIZES], ids=["%s-%d" % (s[0], i) for i, s in enumerate(SIZES)])
def test_wrong_offsets_stay_inside(loads, dropped, width, cols, dtype, act, transposed):
    import paper_2007_14152_amd as sp
    L, n, rows, code = sp.lib(), len(loads), sum(loads) + dropped, TYPES[dtype]
    size, bytes_of = torch.empty(0, dtype=dtype).element_size(), ctypes.c_size_t()
    x, w = torch.ones(rows, width, dtype=dtype, device=DEV), torch.ones(n, width, cols, dtype=dtype, device=DEV)
    dout, pre_in = torch.ones(rows, cols, dtype=dtype, device=DEV), torch.ones(rows, cols, dtype=dtype, device=DEV)
    wstride = width if transposed else cols
    assert L.spdnn_linear_bytes(rows, width, cols, 1, n, code, ctypes.byref(bytes_of)) == 0
    need = bytes_of.value
    assert L.spdnn_linear_grad_bytes(rows, width, cols, 1, n, code, code, act, transposed, ctypes.byref(bytes_of)) == 0
    grad_need = bytes_of.value
    out, pre, dx, dw, db = (Guarded(c, size) for c in (rows * cols, rows * cols, rows * width, n * width * cols, n * cols))
    work, grad_work = Guarded(need, 1), Guarded(grad_need, 1)
    assert work.p % 256 == 0 and grad_work.p % 256 == 0
    stream = torch.cuda.current_stream().cuda_stream
    for at in wrong(rows, n):
        off = torch.tensor(at[:n + 1], dtype=torch.int32, device=DEV)
        assert L.spdnn_linear(x.data_ptr(), code, rows, width, width, off.data_ptr(), n, w.data_ptr(), transposed, wstride, width * cols, cols, 0, 0, act, 0, cols,
                              out.p, code, cols, pre.p, cols, work.p, need, stream) == 0
        for dxp, dwp, dbp in ((dx.p, dw.p, db.p), (0, 0, db.p)):
            assert L.spdnn_linear_grad(dout.data_ptr(), code, cols, pre_in.data_ptr(), cols, act, x.data_ptr(), code, rows, width, width, off.data_ptr(), n, w.data_ptr(),
                                       transposed, wstride, width * cols, cols, dxp, width, dwp, wstride, width * cols, dbp, code, grad_work.p, grad_need, stream) == 0
        torch.cuda.synchronize()
        for what, t in (("out", out), ("pre", pre), ("dx", dx), ("dweight", dw), ("dbias", db), ("work", work), ("work of gradients", grad_work)):
            assert t.whole(), (what, at[:n + 1])


def test_wrong_offsets_of_more_tiles_than_32_bits_hold():
    """1024 experts that all claim all of 2^28 rows."""
    import paper_2007_14152_amd as sp
    L, n, rows = sp.lib(), 1024, 1 << 28
    x, w = torch.ones(rows, 1, dtype=torch.bfloat16, device=DEV), torch.ones(n, 1, 1, dtype=torch.bfloat16, device=DEV)
    need = ctypes.c_size_t()
    assert L.spdnn_linear_bytes(rows, 1, 1, 1, n, 1, ctypes.byref(need)) == 0
    out, work = Guarded(rows, 2), Guarded(need.value, 1)
    for at in ([0, rows] * n, [rows, 0] * n, [0] + [rows] * n):
        off = torch.tensor(at[:n + 1], dtype=torch.int32, device=DEV)
        assert L.spdnn_linear(x.data_ptr(), 1, rows, 1, 1, off.data_ptr(), n, w.data_ptr(), 0, 1, 1, 1, 0, 0, 0, 0, 1, out.p, 1, 1, 0, 1, work.p, need.value,
                              torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert out.whole() and work.whole(), at[:3]
    # the last is right: all rows belong to the first expert
    assert bool((out.t[ROOM:-ROOM].view(torch.bfloat16) == 1).all())

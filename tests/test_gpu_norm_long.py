"""Gradients of layer norm over rows that registers do not hold, in no more work memory than the library asks for."""
import ctypes

import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", [(1, 32769), (40, 33000), (17, 40000), (600, 16385)])
def test_long_rows_stay_in_their_work_memory(rows, width, dtype):
    import paper_2007_14152_amd as sp
    L, g = sp.lib(), torch.Generator().manual_seed(rows)
    x, dout, w = torch.randn(rows, width, generator=g).to(dtype), torch.randn(rows, width, generator=g).to(dtype), torch.randn(width, generator=g)
    xd, dd, wd = x.to(DEV), dout.to(DEV), w.to(DEV)
    stats = sp.layer_norm(xd, wd, stats=True)[1]
    size = ctypes.c_size_t()
    assert L.spdnn_layer_norm_grad_bytes(rows, width, ctypes.byref(size)) == 0
    room = 1 << 16
    work = torch.full((size.value // 4 + 2 * room,), 5.0, device=DEV)
    at = work.data_ptr() + 4 * room
    assert at % 256 == 0
    dx, dw, db = torch.empty_like(xd), torch.empty(width, device=DEV), torch.empty(width, device=DEV)
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype]
    assert L.spdnn_layer_norm_grad(dd.data_ptr(), code, width, xd.data_ptr(), rows, width, width, stats.data_ptr(), wd.data_ptr(), 0, 0, width, dx.data_ptr(), width,
                                   dw.data_ptr(), db.data_ptr(), 0, at, size.value, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert bool((work[:room] == 5).all()) and bool((work[-room:] == 5).all())
    want, off = ref.norm_grad(dout, x, stats.cpu(), w)
    for what, a, b, c in zip(("dx", "dweight", "dbias"), (dx, dw, db), want, off):
        ref.assert_within(a, b.numpy(), c.numpy(), a.dtype, what)

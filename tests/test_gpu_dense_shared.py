"""Dense products of operands whose lines are all one row in memory (stride 0), of odd and even lengths."""
import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def whole(g, shape, dtype):
    return torch.randint(-2, 3, shape, generator=g).to(dtype)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width,cols", [(1, 33, 20), (1, 4097, 300), (2, 1, 9), (70, 33, 20), (70, 64, 20), (5, 777, 300), (300, 777, 129), (257, 65, 300), (3000, 71, 2903), (20, 8201, 64)])
def test_rows_that_are_one(sp, rows, width, cols, dtype, transposed):
    """x, and then dout, with the same row for all."""
    g = torch.Generator().manual_seed(rows + width)
    x, w, dout = whole(g, (1, width), dtype).expand(rows, width), whole(g, (width, cols), dtype), whole(g, (1, cols), dtype).expand(rows, cols)
    wd = w.t().contiguous().to(DEV).t() if transposed else w.to(DEV)
    xd, dd = x[:1].to(DEV).expand(rows, width), dout[:1].to(DEV).expand(rows, cols)
    assert torch.equal(sp.linear(xd, wd, dtype=F32).cpu().double(), x.double() @ w.double())
    dx, dw, db = sp.linear_grad(dd, xd, wd, dtype=F32)
    assert torch.equal(dx.cpu(), (dout.double() @ w.double().t()).to(dtype))
    assert torch.equal(dw.cpu().double(), x.double().t() @ dout.double()) and torch.equal(db.cpu().double(), dout.double().sum(0))
    offsets = torch.tensor([0, rows // 3, rows // 3, rows - 1], dtype=torch.int32)
    ws = whole(g, (3, width, cols), dtype)
    wsd = ws.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) if transposed else ws.to(DEV)
    want, grads = ref.linear(x, ws, offsets=offsets)[0], ref.linear_grad(dout, x, ws, offsets=offsets)[0]
    assert torch.equal(sp.grouped_linear(xd, offsets.to(DEV), wsd, dtype=F32).cpu().double(), want)
    for a, b in zip(sp.grouped_linear_grad(dd, xd, offsets.to(DEV), wsd, dtype=F32), grads):
        assert torch.equal(a.cpu(), b.to(a.dtype))


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width,cols", [(3, 1, 9), (70, 33, 200), (300, 777, 520), (70, 64, 20)])
def test_columns_that_are_one(sp, rows, width, cols, dtype):
    """The same column of W for all, W stored with its rows adjacent, and the same row for all."""
    g = torch.Generator().manual_seed(rows + width)
    x, dout = whole(g, (rows, width), dtype), whole(g, (rows, cols), dtype)
    column, row = whole(g, (1, width), dtype), whole(g, (1, cols), dtype)
    for w, wd in ((column.expand(cols, width).t(), column.to(DEV).expand(cols, width).t()), (row.expand(width, cols), row.to(DEV).expand(width, cols))):
        assert torch.equal(sp.linear(x.to(DEV), wd, dtype=F32).cpu().double(), x.double() @ w.double())
        dx, dw, db = sp.linear_grad(dout.to(DEV), x.to(DEV), wd, dtype=F32)
        assert torch.equal(dx.cpu(), (dout.double() @ w.double().t()).to(dtype)) and torch.equal(dw.cpu().double(), x.double().t() @ dout.double())

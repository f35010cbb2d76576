"""The row operators where their outputs are too large for the caches, and tables that several launches clear together.  Values
are small whole numbers, so that every sum is exact in any order and outputs have to be equal."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def whole(seed, shape, dtype, most=4):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).to(dtype)


def spoil(shape, dtype):
    """Leaves NaN in the memory that the allocator hands out next for such a tensor."""
    torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def some_ids(seed, n, vocab, which):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(-1, vocab, (n,), generator=g, device=DEV)
    if which == "crowded":  # most rows without an id, a few with many
        ids = torch.where(ids % 3 == 0, ids, ids % 50)
    ids[:4] = torch.tensor([0, vocab - 1, vocab // 2, vocab])
    return ids


# Tables of more than the sort clears beside (24 and 40 MB a digit, without the 24 where one chunk holds all ids): the rest is
# cleared by the kernel that adds, between rows that have ids.
TABLES = [(5000, 70001, 1001, F32, F32), (1500, 70001, 501, F32, F32), (5000, 70001, 1003, BF16, BF16), (2049, 50003, 2050, F16, F32),
          (40000, 66000, 1024, BF16, F32), (3000, 1023, 40001, F32, F32), (1025, 60000, 4096, BF16, BF16)]


@pytest.mark.parametrize("which", ["spread", "crowded"])
@pytest.mark.parametrize("n,vocab,width,dtype,otype", TABLES + [(700, 70001, 1001, F32, F32), (1024, 70001, 2047, BF16, BF16), (1, 60000, 4096, BF16, F32)])
def test_gradient_of_a_large_table(sp, n, vocab, width, dtype, otype, which):
    dout, ids = whole(n, (n, width), dtype), some_ids(vocab, max(n, 4), vocab, which)[:n]
    want = torch.zeros(vocab + 1, width, device=DEV).index_add_(0, torch.where(ids < 0, vocab, ids), dout.float())[:vocab]
    spoil((vocab, width), otype)
    assert torch.equal(sp.embed_grad(dout, ids, vocab, dtype=otype), want.to(otype))
    base = whole(3, (vocab, width), otype)
    there = base.clone()
    assert torch.equal(sp.embed_grad(dout, ids, vocab, out=there), (base.float() + want).to(otype))


@pytest.mark.parametrize("n,vocab,width", [(5000, 70001, 600), (1500, 70001, 601), (700, 70001, 599)])
def test_rows_with_gaps_between_them(sp, n, vocab, width):
    """What stands between the rows of a table stays, whichever launch clears the rows."""
    dout, ids = whole(n, (n, width), F32), some_ids(n, n, vocab, "spread")
    want = torch.zeros(vocab + 1, width, device=DEV).index_add_(0, torch.where(ids < 0, vocab, ids), dout)[:vocab]
    wide = torch.full((vocab, width + 3), 7.0, device=DEV)
    size = ctypes.c_size_t()
    assert sp.lib().spdnn_embed_grad_bytes(vocab, width, n, ctypes.byref(size)) == sp.SPDNN_OK
    work = torch.empty(max(size.value, 1), dtype=torch.uint8, device=DEV)
    rc = sp.lib().spdnn_embed_grad(dout.data_ptr(), sp.SPDNN_F32, width, ids.data_ptr(), sp.SPDNN_I64, n, vocab, width, 1.0, 0,
                                   wide.data_ptr() + 4, sp.SPDNN_F32, width + 3, work.data_ptr(), size.value,
                                   torch.cuda.current_stream().cuda_stream)
    assert rc == sp.SPDNN_OK
    assert torch.equal(wide[:, 1:width + 1], want)
    assert (wide[:, 0] == 7).all() and (wide[:, width + 1:] == 7).all()


@pytest.mark.parametrize("n,width,ttype,otype", [(24000, 4096, BF16, BF16), (41000, 1001, F32, F32), (30000, 2777, F16, F16), (15001, 2777, BF16, F32),
                                                 (300000, 139, F32, F32)])
def test_many_rows_of_a_table(sp, n, width, ttype, otype):
    table, ids = whole(1, (5000, width), ttype), some_ids(2, n, 5000, "spread")
    want = torch.where(((ids >= 0) & (ids < 5000))[:, None], 2 * table[ids.clamp(0, 4999)].float(), 0.0).to(otype)
    spoil((n, width), otype)
    assert torch.equal(sp.embed(table, ids, scale=2.0, dtype=otype), want)


@pytest.mark.parametrize("rows,k,width,dtype", [(5001, 4, 2051, F32), (40001, 4, 515, BF16), (81001, 2, 255, F32), (20500, 1, 4097, BF16),
                                                (9001, 5, 2000, F16), (20001, 2, 2051, F32)])
def test_large_batches_there_and_back(sp, rows, k, width, dtype):
    experts = 12
    chosen = torch.randint(-1, experts, (rows, k), generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV, dtype=torch.int32)
    x, ys, dout, add = (whole(s, shape, dtype, 2) for s, shape in ((1, (rows, width)), (2, (rows * k, width)), (3, (rows, width)), (4, (rows, width))))
    weight = whole(5, (rows, k), F32, 3)
    spoil((rows * k, width), dtype)
    xs, offsets, place = sp.dispatch(x, chosen, experts)
    used = int(offsets[-1])
    flat = place.reshape(-1)
    pair = torch.nonzero(flat >= 0)[:, 0]
    at = flat[pair].long()
    assert len(pair) == used and torch.equal(torch.sort(at).values, torch.arange(used, device=DEV))
    want = torch.zeros(rows * k, width, dtype=dtype, device=DEV)
    want[at] = x[pair // k]
    assert torch.equal(xs, want)
    del xs
    # combine: sums of whole numbers of at most 2 + 5 * 6, which every type holds
    total = add.float().clone()
    for j in range(k):
        total += torch.where(place[:, j:j + 1] >= 0, weight[:, j:j + 1] * ys[place[:, j].clamp(min=0).long()].float(), 0.0)
    spoil((rows, width), dtype)
    assert torch.equal(sp.combine(ys, place, weight=weight, add=add), total.to(dtype))
    # combine_grad
    spoil((rows * k, width), dtype)
    dys, dweight = sp.combine_grad(dout, ys, place, weight, offsets)
    want.zero_()
    want[at] = (weight.reshape(-1)[pair][:, None] * dout[pair // k].float()).to(dtype)
    assert torch.equal(dys, want)
    dw = torch.zeros(rows * k, device=DEV)
    dw[pair] = (dout[pair // k].float() * ys[at].float()).sum(1)
    assert torch.equal(dweight.reshape(-1), dw)

"""Dense products and layer norm against their formulas in 64 bits (dense_ref.py), at the sizes, masks and layouts where they can go
wrong; gradients also against differences of the forward operators.  Products of small whole numbers have exact sums: those tests ask
for equality."""
import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = ref.TYPES


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def laid(t, layout):
    """A matrix of rows on the GPU as it is; as part of wider rows, off by one element; its first row for all (stride 0)."""
    if layout == "dense":
        return t.to(DEV)
    if layout == "part":
        wide = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), dtype=t.dtype)
        wide[:, 1:t.shape[1] + 1] = t
        return wide.to(DEV)[:, 1:t.shape[1] + 1]
    return t[:1].to(DEV).expand(t.shape)


def whole(g, shape, dtype, most=2):
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def stored(w, transposed):
    """The same weights on the GPU, stored with their rows adjacent or the other way round."""
    return w.transpose(-1, -2).contiguous().to(DEV).transpose(-1, -2) if transposed else w.to(DEV)


def equal(got, want, what=""):
    want = want.to(got.dtype)
    same = torch.equal(got.cpu(), want)
    assert same, (what, int((got.cpu() != want).sum()), (got.cpu() != want).nonzero()[:4].tolist())


def within(got, want, off, what=""):
    ref.assert_within(got, want.numpy(), off.numpy(), got.dtype, what)


def loads(seed, rows, experts, dropped=0):
    """Offsets of uneven batches, some empty."""
    g = torch.Generator().manual_seed(seed)
    p = torch.rand(experts, generator=g) ** 2 * (torch.rand(experts, generator=g) > 0.2)
    at = torch.cumsum(p, 0)
    at = (at / at[-1].clamp(min=1e-9) * (rows - dropped)).round().long() if rows else torch.zeros(experts, dtype=torch.long)
    return torch.cat([torch.zeros(1, dtype=torch.long), at]).to(torch.int32)


# one token to a few hundred, sizes around a fragment, a step of k, a tile; several tiles; splits
SIZES = [(1, 1, 1), (1, 64, 64), (1, 4096, 64), (2, 7, 5), (3, 33, 130), (15, 32, 16), (16, 31, 17), (17, 64, 100), (33, 65, 63), (64, 128, 128),
         (65, 100, 200), (127, 96, 129), (129, 250, 127), (257, 64, 300), (300, 777, 520), (5, 8200, 96), (1000, 48, 33),
         # chunks of 16 bytes, and steps of k that are not whole
         (40, 72, 136), (130, 1000, 264), (90, 520, 40), (200, 8, 8), (1, 8200, 4104), (20, 136, 4160)]


@pytest.mark.parametrize("layout", ["dense", "part"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width,cols", SIZES)
def test_linear_exact(sp, rows, width, cols, dtype, transposed, layout):
    g = torch.Generator().manual_seed(rows * 1000 + width + cols)
    x, w = whole(g, (rows, width), dtype), whole(g, (width, cols), dtype)
    bias, add = whole(g, (cols,), dtype, 9), whole(g, (rows, cols), dtype, 9)
    got, pre = sp.linear(laid(x, layout), stored(w, transposed), bias=bias.to(DEV), act="clip", add=laid(add, layout), pre=True)
    z = x.double() @ w.double() + bias.double()
    equal(pre, z, "pre")
    equal(got, z.clamp(0, 32) + add.double(), "out")
    equal(sp.linear(laid(x, layout), stored(w, transposed), dtype=F32), x.double() @ w.double(), "plain, to 32 bits")


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width,cols", SIZES)
def test_linear_grad_exact(sp, rows, width, cols, dtype, transposed):
    g = torch.Generator().manual_seed(rows + 1000 * width + cols)
    x, w, dout = whole(g, (rows, width), dtype), whole(g, (width, cols), dtype), whole(g, (rows, cols), dtype)
    pre = whole(g, (rows, cols), dtype, 40)
    for layout, act in (("dense", "clip"), ("part", None), ("dense", None), ("one", "relu")):
        if layout == "one":
            dout = dout[:1].expand(rows, cols)
        d = dout.double() * ref.slope(pre.double(), act)
        dx, dw, db = sp.linear_grad(laid(dout, layout), laid(x, "part" if layout == "part" else "dense"), stored(w, transposed),
                                    pre=laid(pre, "part") if act else None, act=act, dtype=F32)
        equal(dx, d @ w.double().t(), "dx")
        equal(dw, x.double().t() @ d, "dweight")
        equal(db, d.sum(0), "dbias")
        assert dw.dtype == db.dtype == F32 and dx.dtype == dtype
        assert dw.transpose(0, 1).is_contiguous() if transposed else dw.is_contiguous()
    part = sp.linear_grad(laid(dout, "one"), x.to(DEV), stored(w, transposed), for_x=False, for_bias=False)
    assert part[0] is None and part[2] is None
    equal(part[1], x.double().t() @ dout.double())


# many tiles: more rows and columns than 256 CUs take at a time in tiles of 128
MANY = [(2900, 200, 2904), (2905, 136, 3000), (8200, 24, 1100), (1030, 328, 8136), (2900, 77, 2903)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width,cols", MANY)
def test_many_tiles_exact(sp, rows, width, cols, dtype, transposed):
    g = torch.Generator().manual_seed(rows + width + cols)
    x, w, bias = whole(g, (rows, width), dtype), whole(g, (width, cols), dtype), whole(g, (cols,), dtype, 9)
    equal(sp.linear(x.to(DEV), stored(w, transposed), bias=bias.to(DEV), act="relu"), (x.double() @ w.double() + bias.double()).clamp(min=0), "out")
    # the same numbers as a gradient: of W [cols, rows], whose batch is the width
    d, y = x.t().contiguous(), w
    dw = sp.linear_grad(y.to(DEV), d.to(DEV), stored(whole(g, (rows, cols), dtype), transposed), dtype=F32, for_x=False, for_bias=False)[1]
    equal(dw, d.double().t() @ y.double(), "dweight")
    dx = sp.linear_grad(x.to(DEV), torch.zeros(rows, cols, dtype=dtype, device=DEV), stored(w.t().contiguous(), transposed), for_weight=False)[0]
    equal(dx, x.double() @ w.double(), "dx")


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_many_grouped_tiles_exact(sp, dtype, transposed):
    g = torch.Generator().manual_seed(6)
    rows, experts, width, cols = 9000, 5, 104, 1800
    offsets = torch.tensor([0, 3000, 3000, 3007, 6500, 8800], dtype=torch.int32)
    x, w, dout = whole(g, (rows, width), dtype), whole(g, (experts, width, cols), dtype), whole(g, (rows, cols), dtype)
    want, grads = ref.linear(x, w, offsets=offsets)[0], ref.linear_grad(dout, x, w, offsets=offsets)[0]
    x[8800:], dout[8800:] = float("nan"), float("nan")
    equal(sp.grouped_linear(x.to(DEV), offsets.to(DEV), stored(w, transposed)), want)
    for what, a, b in zip(("dx", "dweight", "dbias"), sp.grouped_linear_grad(dout.to(DEV), x.to(DEV), offsets.to(DEV), stored(w, transposed), dtype=F32), grads):
        equal(a, b, what)


GROUPS = [(1, 2, 64, 64, 0), (8, 256, 64, 80, 0), (40, 3, 33, 50, 7), (256, 64, 128, 64, 20), (300, 5, 65, 130, 0), (513, 300, 40, 24, 100),
          (700, 2, 64, 256, 700), (900, 7, 96, 31, 1), (64, 1024, 16, 16, 0), (0, 4, 32, 32, 0), (1500, 4, 200, 136, 3)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,experts,width,cols,dropped", GROUPS)
def test_grouped_exact(sp, rows, experts, width, cols, dropped, dtype, transposed):
    g = torch.Generator().manual_seed(rows + experts)
    offsets = loads(rows, rows, experts, dropped)
    used = int(offsets[-1])
    x, w = whole(g, (rows, width), dtype), whole(g, (experts, width, cols), dtype)
    bias, add, pre, dout = whole(g, (experts, cols), dtype, 9), whole(g, (rows, cols), dtype, 9), whole(g, (rows, cols), dtype, 40), whole(g, (rows, cols), dtype)
    want, _, z, _ = ref.linear(x, w, bias, "relu", add, offsets)
    plain = ref.linear(x, w, offsets=offsets)[0]
    grads = ref.linear_grad(dout, x, w, pre, "clip", offsets)[0]
    grads_plain = ref.linear_grad(dout, x, w, offsets=offsets)[0]
    for t in (x, add, pre, dout):  # what rows of no expert hold does not matter
        t[used:] = float("nan")
    off = offsets.to(DEV)
    for layout in ("dense", "part"):
        got, before = sp.grouped_linear(laid(x, layout), off, stored(w, transposed), bias=bias.to(DEV), act="relu", add=laid(add, layout), pre=True)
        equal(got, want, "out")
        equal(before, z, "pre")
        equal(sp.grouped_linear(laid(x, layout), off, stored(w, transposed), dtype=F32), plain, "plain")
        for what, got, want_grad in zip(("dx", "dweight", "dbias"), sp.grouped_linear_grad(laid(dout, layout), laid(x, layout), off, stored(w, transposed),
                                        pre=laid(pre, layout), act="clip", dtype=F32), grads):
            equal(got, want_grad, what)
        for what, got, want_grad in zip(("dx", "dweight", "dbias"), sp.grouped_linear_grad(laid(dout, layout), laid(x, layout), off, stored(w, transposed)),
                                        grads_plain):
            equal(got, want_grad, what)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,experts", [(1, 1), (2, 2), (3, 2), (15, 16), (16, 16), (17, 16), (18, 16), (64, 64), (68, 64), (69, 64), (256, 256), (272, 256),
                                          (273, 256), (274, 256), (290, 256), (1024, 1024), (1090, 1024), (1100, 1024),
                                          # and experts about as many as a wave has lanes
                                          (100, 63), (130, 65), (127, 127), (500, 128), (9000, 63), (9000, 64), (20000, 130)])
def test_about_as_many_rows_as_experts(sp, rows, experts, dtype):
    """Every row in a tile of its own or all in one, whatever the tiles are counted by; out of memory that held something else."""
    g = torch.Generator().manual_seed(rows + experts)
    x, w, dout = whole(g, (rows, 24), dtype), whole(g, (experts, 24, 40), dtype), whole(g, (rows, 40), dtype)
    at = torch.arange(experts + 1)
    for offsets in (at.clamp(max=rows), at.clamp(max=rows - 1), (at - experts + rows).clamp(0, rows) * at.sign(), at.sign() * rows, at // experts * rows, at * 0,
                    loads(1, rows, experts)):
        offsets = offsets.to(torch.int32)
        want, grads = ref.linear(x, w, offsets=offsets)[0], ref.linear_grad(dout, x, w, offsets=offsets)[0]
        off = offsets.to(DEV)
        torch.full((rows, 40), float("nan"), dtype=dtype, device=DEV)
        equal(sp.grouped_linear(x.to(DEV), off, w.to(DEV)), want)
        for what, a, b in zip(("dx", "dweight", "dbias"), sp.grouped_linear_grad(dout.to(DEV), x.to(DEV), off, w.to(DEV), dtype=F32), grads):
            equal(a, b, what)


@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("rows,width,cols", [(1, 300, 77), (37, 128, 64), (200, 520, 264)])
def test_linear_of_real_numbers(sp, rows, width, cols, dtype, out, name):
    g = torch.Generator().manual_seed(rows)
    x, w = normal(g, (rows, width), dtype), normal(g, (width, cols), dtype, 2 / width ** 0.5)
    bias, add = normal(g, (cols,), F32, 3), normal(g, (rows, cols), out)
    got, pre = sp.linear(x.to(DEV), w.to(DEV), bias=bias.to(DEV), act=name, add=add.to(DEV), pre=True, dtype=out)
    want, off, z, zoff = ref.linear(x, w, bias, name, add)
    within(pre, z, zoff, "pre")
    within(got, want, off, "out")
    dout = normal(g, (rows, cols), out)
    grads = sp.linear_grad(dout.to(DEV), x.to(DEV), w.to(DEV), pre=pre, act=name)
    want, off = ref.linear_grad(dout, x, w, pre.cpu(), name)
    for what, a, b, c in zip(("dx", "dweight", "dbias"), grads, want, off):
        within(a, b, c, what)
        assert a.dtype == dtype


@pytest.mark.parametrize("name", ref.ACTS)
def test_linear_grad_against_differences(sp, name):
    g = torch.Generator().manual_seed(5)
    rows, width, cols, offsets = 40, 24, 30, torch.tensor([0, 13, 13, 37], dtype=torch.int32)
    x, w, b = normal(g, (rows, width), F32), normal(g, (3, width, cols), F32, 0.4), normal(g, (3, cols), F32)
    dout = normal(g, (rows, cols), F32)
    off = offsets.to(DEV)
    out, pre = sp.grouped_linear(x.to(DEV), off, w.to(DEV), bias=b.to(DEV), act=name, pre=True)
    grads = sp.grouped_linear_grad(dout.to(DEV), x.to(DEV), off, w.to(DEV), pre=pre, act=name)
    h = 2.0 ** -10
    for i, t in enumerate((x, w, b)):
        step = normal(g, t.shape, F32)
        def at(sign):
            args = [x, w, b]
            args[i] = t + sign * h * step
            return sp.grouped_linear(args[0].to(DEV), off, args[1].to(DEV), bias=args[2].to(DEV), act=name).cpu().double()
        change = ((at(1) - at(-1)) / (2 * h))[:37]
        got = float((grads[i].cpu().double() * step.double()).sum())
        # 32-bit outputs are off by their bound each; gelu and silu have third derivatives below 2, and relu and clip have corners, left
        # out where a corner lies between the two points
        z, zoff = ref.linear(x, w, b, None, None, offsets)[2:]
        far = torch.zeros_like(z)
        for e, lo, hi in ref.batches(rows, offsets):
            far[lo:hi] = {0: lambda: step[lo:hi].double() @ w[e].double(), 1: lambda: x[lo:hi].double() @ step[e].double(),
                          2: lambda: step[e].double().expand(hi - lo, cols)}[i]()
        far, z, zoff, d = far[:37], z[:37], zoff[:37], dout.double()[:37]
        smooth = torch.ones_like(z, dtype=torch.bool)
        if name in ("relu", "clip"):
            smooth = (z.abs() > h * far.abs() + zoff) & ((z - 32).abs() > h * far.abs() + zoff)
        want = float((d * change)[smooth].sum()) + float((d * ref.slope(z, name) * far)[~smooth].sum())
        room = float((d.abs() * ((2.26 * zoff + 2 * ref.act_off(z, name) + ref.U * ref.act(z, name).abs()) / h + h * h / 3 * far.abs() ** 3)).sum())
        room += float((ref.linear_grad(dout, x, w, pre.cpu(), name, offsets)[1][i] * step.double().abs()).sum())
        assert abs(got - want) <= room, (i, got, want, room)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_linear_special_numbers(sp, dtype):
    """A NaN or an infinity stays in the rows and columns that it belongs to, whatever the sizes leave over in a tile."""
    g = torch.Generator().manual_seed(2)
    x, w = whole(g, (70, 50), dtype, 1).abs() + 1, whole(g, (50, 40), dtype, 1).abs() + 1
    x[3, 49], x[69, 0], w[49, 39] = float("nan"), float("inf"), float("inf")
    out = sp.linear(x.to(DEV), w.to(DEV)).cpu()
    want = x.double() @ w.double()
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.isinf(), want.isinf())
    fin = want.isfinite()
    assert torch.equal(out[fin], want.to(dtype)[fin])
    assert sp.linear(x.to(DEV), w.to(DEV), act="relu").cpu()[3].isnan().all()
    assert sp.linear(x.to(DEV), w.to(DEV), act="clip").cpu()[3].isnan().all()
    dx, dw, db = sp.linear_grad(torch.ones(70, 40, dtype=dtype, device=DEV), x.to(DEV), w.to(DEV))
    assert dw.cpu()[49].isnan().all() and dw.cpu()[0].isinf().all() and dw.cpu()[1:49].isfinite().all()
    assert dx.cpu()[:, 49].isinf().all() and dx.cpu()[:, :49].isfinite().all() and db.cpu().isfinite().all()


def test_linear_without_rows(sp):
    for dtype in ref.TYPES:
        x, w = torch.empty(0, 24, dtype=dtype, device=DEV), torch.ones(24, 40, dtype=dtype, device=DEV)
        assert sp.linear(x, w, act="gelu").shape == (0, 40)
        dx, dw, db = sp.linear_grad(torch.empty(0, 40, dtype=dtype, device=DEV), x, w)
        assert dx.shape == (0, 24) and not dw.any() and not db.any() and dw.shape == (24, 40)
        off = torch.zeros(3, dtype=torch.int32, device=DEV)
        y = sp.grouped_linear(torch.full((9, 24), float("nan"), dtype=dtype, device=DEV), off, w.expand(2, 24, 40))
        assert y.shape == (9, 40) and not y.any()
        dx, dw, db = sp.grouped_linear_grad(torch.full((9, 40), float("nan"), dtype=dtype, device=DEV), torch.full((9, 24), float("nan"), dtype=dtype, device=DEV),
                                            off, w.expand(2, 24, 40))
        assert not dx.any() and not dw.any() and not db.any()


def test_offsets_that_do_not_ascend_stay_inside(sp):
    """Nothing outside the arrays is touched; the rows themselves are not specified."""
    x, w = torch.ones(200, 32, device=DEV), torch.ones(4, 32, 48, device=DEV)
    for at in ([0, 300, 50, 900, 200], [-5, -9, 2 ** 31 - 1, -2 ** 31, 7], [200, 150, 100, 50, 0], [7, 7, 7, 7, 7]):
        off = torch.tensor(at, dtype=torch.int32, device=DEV)
        guard = torch.full((3 * 200, 48), 5.0, device=DEV)
        out = sp.grouped_linear(x, off, w)
        assert out.shape == (200, 48)
        sp.grouped_linear_grad(torch.ones(200, 48, device=DEV), x, off, w)
        assert bool((guard == 5).all())


def test_linear_one_by_many_strides(sp):
    """Weights with a stride between their rows, one matrix for all experts, rows far apart."""
    g = torch.Generator().manual_seed(9)
    for dtype in ref.TYPES:
        x, w = whole(g, (150, 72), dtype), whole(g, (72, 88), dtype)
        wide = torch.full((72, 100), float("nan"), dtype=dtype, device=DEV)
        wide[:, 4:92] = w.to(DEV)
        want = x.double() @ w.double()
        equal(sp.linear(x.to(DEV), wide[:, 4:92]), want)
        off = torch.tensor([0, 20, 150], dtype=torch.int32, device=DEV)
        equal(sp.grouped_linear(x.to(DEV), off, w.to(DEV).expand(2, 72, 88)), want)
        dx, dw, db = sp.grouped_linear_grad(want.sign().to(dtype).to(DEV), x.to(DEV), off, wide[:, 4:92].expand(2, 72, 88))
        d = want.sign()
        equal(dx, d @ w.double().t())
        equal(dw, torch.stack([x[:20].double().t() @ d[:20], x[20:].double().t() @ d[20:]]))
        one = whole(g, (1, 88), dtype)  # a weight that is one row for all
        equal(sp.linear(x.to(DEV), one.to(DEV).expand(72, 88)), x.double() @ one.double().expand(72, 88))


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------
WIDTHS = [(1, 1), (3, 2), (5, 7), (9, 8), (70, 64), (6, 100), (130, 513), (4, 1500), (33, 2048), (5, 4097), (3, 8200), (2, 16384), (2, 20001), (2, 70000), (700, 24)]


@pytest.mark.parametrize("layout", ["dense", "part"])
@pytest.mark.parametrize("dtype,out,param", [(F32, F32, F32), (BF16, BF16, BF16), (F16, F16, F32), (BF16, F32, F32)])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_layer_norm(sp, rows, width, dtype, out, param, layout):
    g = torch.Generator().manual_seed(rows + width)
    x = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(width, generator=g) * 0.5) + torch.randn(rows, 1, generator=g) * 3).to(dtype)
    w, b = normal(g, (width,), param) + 1, normal(g, (width,), param)
    got, stats = sp.layer_norm(laid(x, layout), w.to(DEV), b.to(DEV), eps=1e-3, stats=True, dtype=out)
    want, off, mean, rstd, mean_off, rstd_off = ref.norm(x, w, b, 1e-3)
    within(got, want, off)
    within(stats[:, :1], mean, mean_off, "mean")
    within(stats[:, 1:], rstd, rstd_off, "rstd")
    want, off = ref.norm(x, eps=1e-3)[:2]
    within(sp.layer_norm(laid(x, layout), eps=1e-3), want, off)
    dout, add = normal(g, (rows, width), dtype), normal(g, (rows, width), dtype)
    want, off = ref.norm_grad(dout, x, stats.cpu(), w, add)
    got = sp.layer_norm_grad(laid(dout, layout), laid(x, layout), stats, w.to(DEV), add=laid(add, layout), dtype=F32)
    for what, a, c, d in zip(("dx", "dweight", "dbias"), got, want, off):
        within(a, c, d, what)
    want, off = ref.norm_grad(dout, x, stats.cpu())
    got = sp.layer_norm_grad(laid(dout, layout), laid(x, layout), stats, for_weight=False)
    assert got[1] is None
    within(got[0], want[0], off[0])
    within(got[2], want[2], off[2])


def test_layer_norm_of_many_rows(sp):
    g = torch.Generator().manual_seed(4)
    for rows, width, dtype in ((5000, 40, BF16), (3001, 264, F32), (2100, 1032, F16)):
        x, dout = normal(g, (rows, width), dtype), normal(g, (rows, width), dtype)
        w = normal(g, (width,), dtype)
        out, stats = sp.layer_norm(x.to(DEV), w.to(DEV), stats=True)
        want, off = ref.norm(x, w)[:2]
        within(out, want, off)
        want, off = ref.norm_grad(dout, x, stats.cpu(), w)
        for a, c, d in zip(sp.layer_norm_grad(dout.to(DEV), x.to(DEV), stats, w.to(DEV)), want, off):
            within(a, c, d)
            assert a.dtype == dtype


def test_layer_norm_special_rows(sp):
    for dtype in ref.TYPES:
        x = torch.ones(6, 40, dtype=dtype)
        x[1] = 1000.0  # no variance
        x[2, 5], x[3, 6] = float("nan"), float("inf")
        x[4] = torch.arange(40).to(dtype)
        out, stats = sp.layer_norm(x.to(DEV), stats=True)
        out = out.cpu()
        assert not out[:2].any() and out[2].isnan().all() and out[3].isnan().all() and out[4:].isfinite().all()
        assert float(stats[0, 1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
        assert sp.layer_norm(x[:0].to(DEV)).shape == (0, 40)
        dx, dw, db = sp.layer_norm_grad(x[:0].to(DEV), x[:0].to(DEV), stats[:0], torch.ones(40, dtype=dtype, device=DEV))
        assert dx.shape == (0, 40) and not dw.any() and not db.any()


def test_layer_norm_grad_against_differences(sp):
    g = torch.Generator().manual_seed(8)
    rows, width, h = 12, 96, 2.0 ** -9
    x, w, b, dout = normal(g, (rows, width), F32), normal(g, (width,), F32), normal(g, (width,), F32), normal(g, (rows, width), F32)
    out, stats = sp.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), stats=True)
    grads = sp.layer_norm_grad(dout.to(DEV), x.to(DEV), stats, w.to(DEV))
    off = ref.norm(x, w, b)[1]
    grad_off = ref.norm_grad(dout, x, stats.cpu(), w)[1]
    for i, t in enumerate((x, w, b)):
        step = normal(g, t.shape, F32)
        def at(sign):
            args = [x, w, b]
            args[i] = t + sign * h * step
            return sp.layer_norm(args[0].to(DEV), args[1].to(DEV), args[2].to(DEV)).cpu().double()
        want = float((dout.double() * (at(1) - at(-1)) / (2 * h)).sum())
        got = float((grads[i].cpu().double() * step.double()).sum())
        room = float((dout.double().abs() * (off * 1.1 + ref.U * out.cpu().double().abs()) / h).sum()) + float((grad_off[i] * step.double().abs()).sum())
        room += float((ref.U * t.double().abs()).max()) / h * float(grads[i].double().abs().sum())  # the arguments are rounded
        if i == 0:  # third derivative along the step: rows of unit variance, |step| about sqrt(width): below 15 |step|^3 / width |w dout|
            size = step.double().norm(dim=1, keepdim=True)
            room += float((h * h / 6 * 15 * (size / width ** 0.5) ** 3 * (dout.double() * w.double()).abs().sum(1, keepdim=True) * 4).sum())
        assert abs(got - want) <= room, (i, got, want, room)

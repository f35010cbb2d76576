"""The row operators against plain implementations in 64 bits (rows_ref.py), at the sizes, masks and layouts where they can
go wrong; gradients also against differences of the forward operators."""
import numpy as np
import pytest
import torch

import rows_ref as ref

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


def normal(seed, shape, dtype, layout="dense", scale=1.0):
    """Rows of a layout: dense; part of wider rows, off by one element; one row for all (stride 0)."""
    g = torch.Generator().manual_seed(seed)
    n, w = shape
    if layout == "dense":
        return (torch.randn(n, w, generator=g) * scale).to(dtype).to(DEV)
    if layout == "part":
        return (torch.randn(n, w + 3, generator=g) * scale).to(dtype).to(DEV)[:, 1:w + 1]
    return (torch.randn(1, w, generator=g) * scale).to(dtype).to(DEV).expand(n, w)


def zipf(seed, n, vocab, dtype=torch.int32, padding=True):
    rng = np.random.default_rng(seed)
    ids = np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)) - 1, vocab - 1).astype(np.int64)
    if padding:
        ids[rng.random(n) < 0.1] = -1
    return torch.from_numpy(ids).to(dtype).to(DEV)


# ---------------------------------------------------------------------------
# embed
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["dense", "part"])
@pytest.mark.parametrize("ttype,otype", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("n,vocab,width", [(1, 1, 1), (1, 50, 1024), (3, 7, 7), (65, 100, 64), (130, 1000, 777), (513, 33, 1500),
                                           (7, 3, 8193), (2000, 500, 8)])
def test_embed(sp, n, vocab, width, ttype, otype, layout):
    table = normal(n + width, (vocab, width), ttype, layout)
    ids = zipf(n, n, vocab, torch.int64 if n % 2 else torch.int32)
    got = sp.embed(table, ids, scale=0.7, dtype=otype)
    i = ids.long().cpu()
    want = (table.cpu().float()[i.clamp(min=0)] * np.float32(0.7)).to(otype)  # one product of 32 bits, rounded once: equal
    want[i < 0] = 0
    assert torch.equal(got.cpu(), want)


def test_embed_ids_outside_the_table(sp):
    table = normal(1, (10, 40), F32)
    for ids in (torch.tensor([-1, 10, 9, -2 ** 31, 2 ** 31 - 1, 0], dtype=torch.int32),
                torch.tensor([-1, 10, 9, -2 ** 63, 2 ** 63 - 1, 2 ** 32, 2 ** 32 + 1, 0], dtype=torch.int64)):
        got = sp.embed(table, ids.to(DEV)).cpu()
        for t, i in enumerate(ids.tolist()):
            want = table[i].cpu() if 0 <= i < 10 else torch.zeros(40)
            assert torch.equal(got[t], want), i


def test_embed_keeps_the_shape_of_ids(sp):
    table = normal(1, (10, 40), BF16)
    ids = torch.arange(6, device=DEV).reshape(2, 3)
    assert sp.embed(table, ids).shape == (2, 3, 40)
    assert torch.equal(sp.embed(table, ids.t()), table[ids.t()])  # ids of any order
    assert sp.embed(table, ids[:0]).shape == (0, 3, 40)
    special = table.clone()
    special[3] = float("nan")
    special[4] = float("inf")
    got = sp.embed(special, ids).reshape(6, 40)
    assert torch.isnan(got[3]).all() and torch.isinf(got[4]).all() and torch.equal(got[:3], special[:3])


def test_rows_beyond_32_bits(sp):
    """Tables and batches of more than 2^32 elements: the last rows are where they belong."""
    vocab, stride = 66000, 65600
    big = torch.empty(vocab * stride, dtype=BF16, device=DEV)
    table = big.view(vocab, stride)[:, 5:77]
    table[[0, 1, vocab - 1]] = normal(3, (3, 72), BF16)
    ids = torch.tensor([vocab - 1, 0, 1], device=DEV)
    assert torch.equal(sp.embed(table, ids), table[ids])
    before = table[[0, 1, vocab - 1]].clone()
    g = normal(4, (3, 72), BF16)
    sp.embed_grad(g, ids, vocab, out=table)
    assert torch.equal(table[ids], (before[[2, 0, 1]].float() + g.float()).to(BF16))
    # dispatch and back: 2 x 33000 rows of 65600
    rows = 33000
    x = big[:rows * stride].view(rows, stride)
    x[:, 0] = torch.arange(rows, device=DEV) % 251
    x[:, -1] = torch.arange(rows, device=DEV) % 241
    chosen = torch.zeros(rows, 2, dtype=torch.int32, device=DEV)
    chosen[:, 1] = 1
    xs, offsets, place = sp.dispatch(x, chosen, 2)
    assert offsets.tolist() == [0, rows, 2 * rows]
    want = torch.arange(rows, device=DEV)
    for half in (xs[:rows], xs[rows:]):
        assert torch.equal(half[:, 0], (want % 251).to(BF16)) and torch.equal(half[:, -1], (want % 241).to(BF16))
    out = sp.combine(xs, place)
    assert torch.equal(out[:, 0], (2 * (want % 251)).to(BF16)) and torch.equal(out[:, -1], (2 * (want % 241)).to(BF16))


# ---------------------------------------------------------------------------
# embed_grad
# ---------------------------------------------------------------------------
GRAD_SIZES = [(0, 5, 16), (1, 1, 1), (1, 40, 9), (2, 3, 1024), (64, 20, 65), (65, 700, 31), (255, 1, 130), (256, 256, 8), (257, 9, 777),
              (1000, 3000, 33), (1025, 10, 257), (4097, 100, 40), (5000, 70000, 5)]


@pytest.mark.parametrize("dtype,otype,layout,ids", [(F32, F32, "dense", torch.int32), (BF16, F32, "part", torch.int64),
                                                    (BF16, BF16, "dense", torch.int64), (F16, F16, "part", torch.int32),
                                                    (F32, BF16, "one", torch.int32)])
@pytest.mark.parametrize("n,vocab,width", GRAD_SIZES)
def test_embed_grad(sp, n, vocab, width, dtype, otype, layout, ids):
    dout = normal(n + vocab, (n, width), dtype, layout)
    at = zipf(n + width, n, vocab, ids)
    got = sp.embed_grad(dout, at, vocab, scale=1.5, dtype=otype)
    want, bound = ref.embed_grad(ref.f64(dout), at.cpu().numpy(), vocab, 1.5)
    ref.assert_within(got, want, bound, otype)
    assert torch.equal(got, sp.embed_grad(dout, at, vocab, scale=1.5, dtype=otype))  # the order of the sum is fixed


@pytest.mark.parametrize("otype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,width", GRAD_SIZES)
def test_embed_grad_adds_to_what_is_there(sp, n, vocab, width, otype):
    dout = normal(n + vocab, (n, width), BF16)
    at = zipf(n + width, n, vocab)
    wide = normal(9, (vocab, width + 2), otype)
    wide[:, 0] = float("nan")  # beside the rows: not touched
    out = wide[:, 1:width + 1]
    before = wide.clone()
    want, bound = ref.embed_grad(ref.f64(dout), at.cpu().numpy(), vocab, -0.5, base=ref.f64(out))
    assert sp.embed_grad(dout, at, vocab, scale=-0.5, out=out) is out
    ref.assert_within(out, want, bound, otype)
    untouched = torch.ones(vocab, dtype=torch.bool)
    untouched[at[at >= 0].long().cpu()] = False
    assert torch.equal(wide[untouched.to(DEV)][:, 1:], before[untouched.to(DEV)][:, 1:])
    assert torch.isnan(wide[:, 0]).all() and torch.equal(wide[:, -1], before[:, -1])


@pytest.mark.parametrize("n", [1, 100, 3000, 20000])
@pytest.mark.parametrize("which", ["one id", "all padding", "first and last", "all different"])
def test_embed_grad_ids_that_gather(sp, which, n):
    vocab, width = 30000, 24
    rng = np.random.default_rng(n)
    ids = {"one id": np.full(n, 17), "all padding": np.where(np.arange(n) % 2, -1, vocab),
           "first and last": np.where(rng.random(n) < 0.5, 0, vocab - 1), "all different": rng.permutation(vocab)[:n]}[which]
    # small whole numbers: every sum is exact, in any order
    dout = torch.from_numpy(rng.integers(-4, 5, (n, width))).float().to(DEV)
    got = sp.embed_grad(dout, torch.from_numpy(ids).to(DEV), vocab)
    want, _ = ref.embed_grad(ref.f64(dout), ids, vocab, 1.0)
    assert np.array_equal(ref.f64(got), want)


@pytest.mark.parametrize("n,vocab,width", [(300000, 1 << 20, 3), (270000, 1000, 8), (2049, (1 << 21) + 5, 1), (1024, 3, 70000),
                                           (1025, 3, 70000), (70000, 40, 12)])
def test_embed_grad_large(sp, n, vocab, width):
    """More chunks than one workgroup adds up at once, three digits, rows longer than a tile, runs of thousands.  Whole numbers:
    every sum is exact."""
    g = torch.Generator().manual_seed(n)
    dout = torch.randint(-4, 5, (n, width), generator=g).float()
    ids = torch.randint(-1, vocab, (n,), generator=g)
    ids[: n // 3] = vocab // 2
    want = torch.zeros(vocab + 1, width, dtype=torch.float64).index_add_(0, torch.where(ids < 0, vocab, ids), dout.double())
    got = sp.embed_grad(dout.to(DEV), ids.to(DEV), vocab)
    assert torch.equal(got.cpu().double(), want[:vocab])


@pytest.mark.parametrize("rows,k,experts,width", [(140000, 2, 1024, 2), (60000, 5, 7, 4), (1, 16, 16, 40000), (64, 16, 64, 9000), (65, 16, 64, 9000)])
def test_dispatch_and_combine_large(sp, rows, k, experts, width):
    """Chunks longer than the least, rows longer than a tile, both sides of the single launch's limit."""
    chosen = pairs(rows, rows, k, experts)
    x = torch.randint(-9, 10, (rows, width), generator=torch.Generator().manual_seed(1)).float().to(DEV)
    xs, offsets, place = sp.dispatch(x, chosen, experts)
    want_place, want_offsets = ref.sort_pairs(chosen.cpu().numpy(), experts)
    assert np.array_equal(place.cpu().numpy(), want_place) and np.array_equal(offsets.cpu().numpy(), want_offsets)
    used = int(want_offsets[-1])
    assert not xs[used:].any()
    there = (place >= 0).sum(1, keepdim=True)
    assert torch.equal(sp.dispatch_grad(xs, place), x * there)  # whole numbers: exact
    dys, dweight = sp.combine_grad(x, xs, place, torch.full((rows, k), 2.0, device=DEV), offsets)
    assert torch.equal(dys, 2 * xs)
    assert torch.equal(dweight, torch.where(place >= 0, (x * x).sum(1, keepdim=True), 0.0))


def test_embed_grad_leaves_masked_rows_out(sp):
    """What stands in rows of padding does not matter, and an id's infinity stays with it."""
    dout = normal(1, (300, 20), F32)
    ids = zipf(2, 300, 50)
    clean = sp.embed_grad(dout, ids, 50)
    dout[ids < 0] = float("nan")
    assert torch.equal(sp.embed_grad(dout, ids, 50), clean)
    first = int(ids[ids >= 0][0])
    dout[torch.nonzero(ids == first)[0, 0], 3] = float("inf")
    got = sp.embed_grad(dout, ids, 50)
    assert torch.isinf(got[first, 3]) and torch.isinf(got).sum() == 1 and not torch.isnan(got).any()


def test_embed_grad_against_differences(sp):
    """embed is linear in the table: with whole numbers <dout, embed(T + V) - embed(T)> equals <embed_grad, V> exactly."""
    rng = np.random.default_rng(5)
    whole = lambda *shape: torch.from_numpy(rng.integers(-3, 4, shape)).float().to(DEV)
    table, v, dout, ids = whole(40, 30), whole(40, 30), whole(500, 30), zipf(3, 500, 40)
    diff = (dout.double() * (sp.embed(table + v, ids, scale=2.0) - sp.embed(table, ids, scale=2.0)).double()).sum()
    assert float(diff) == float((sp.embed_grad(dout, ids, 40, scale=2.0).double() * v.double()).sum())


# ---------------------------------------------------------------------------
# route
# ---------------------------------------------------------------------------
ROUTE_SIZES = [(1, 1, 1), (1, 2, 2), (5, 3, 2), (64, 8, 2), (3, 16, 16), (33, 63, 4), (17, 64, 8), (9, 65, 3), (40, 100, 16), (130, 128, 1),
               (31, 256, 8), (2, 257, 16), (7, 1000, 5), (4, 1024, 16)]
SCORES = [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)]


def router_input(seed, rows, experts, dtype, layout, with_bias, masked):
    logits = normal(seed, (rows, experts), dtype, layout, scale=2.0)
    if masked and layout != "one":
        g = torch.Generator().manual_seed(seed + 1)
        off = (torch.rand(rows, experts, generator=g) < 0.3).to(DEV)
        logits[off] = -float("inf")
        logits[:, ::7] = torch.finfo(dtype).min  # closed by the type's lowest value: still open, but last
        logits[:: 5] = torch.where(off[::5], float("nan"), logits[::5])
    g = torch.Generator().manual_seed(seed + 2)
    bias = torch.randn(experts, generator=g).to(DEV) if with_bias else None
    keep = (torch.rand(rows, generator=g) < 0.8).to(DEV) if masked else None
    return logits, bias, keep


def check_route(got, logits, k, bias, keep, score, normalise, scale):
    l32 = logits.float().cpu().numpy()
    chosen, is_open = ref.choose(l32, k, None if bias is None else bias.cpu().numpy(), None if keep is None else keep.cpu().numpy())
    assert np.array_equal(got[0].cpu().numpy(), chosen)
    l = np.where(is_open, l32.astype(np.float64), -np.inf)
    want = ref.weights(l, is_open, chosen, score, normalise, scale)
    ref.assert_within(got[1], want, np.abs(want) * ref.weight_slack(l, is_open, l.shape[1]), F32)
    return chosen, is_open, l


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,layout,with_bias", [(F32, "dense", False), (BF16, "part", True), (F16, "dense", True), (F32, "one", True)])
@pytest.mark.parametrize("score,normalise", SCORES)
@pytest.mark.parametrize("rows,experts,k", ROUTE_SIZES)
def test_route_and_gradient(sp, rows, experts, k, score, normalise, dtype, layout, with_bias, masked):
    logits, bias, keep = router_input(rows + experts, rows, experts, dtype, layout, with_bias, masked)
    got = sp.route(logits, k, bias=bias, keep=keep, score=score, normalise=normalise, scale=2.5)
    chosen, is_open, l = check_route(got, logits, k, bias, keep, score, normalise, 2.5)
    dw = normal(k, (rows, k), F32).contiguous()
    dw[got[0] < 0] = float("nan")  # not used
    d = sp.route_grad(dw, logits, got[0], bias=bias, score=score, normalise=normalise, scale=2.5)
    want, bound = ref.route_grad(ref.f64(dw), l, is_open, chosen, score, normalise, 2.5)
    ref.assert_within(d, want, bound, dtype)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_route_takes_the_first_of_equals(sp, dtype):
    for rows, experts, k in [(3, 8, 3), (5, 64, 8), (2, 300, 16)]:
        logits = torch.zeros(rows, experts, dtype=dtype, device=DEV)
        logits[1, ::2] = -0.0  # equal to 0
        assert torch.equal(sp.route(logits, k)[0].cpu(), torch.arange(k, dtype=torch.int32).expand(rows, k))
        few = torch.randint(-2, 3, (rows, experts), generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
        want, _ = ref.choose(few.float().cpu().numpy(), k)
        assert np.array_equal(sp.route(few, k)[0].cpu().numpy(), want)


def test_route_without_rows(sp):
    none = torch.empty(0, 12, device=DEV)
    chosen, weight = sp.route(none, 3)
    assert chosen.shape == (0, 3) and weight.shape == (0, 3)
    assert sp.route_grad(weight, none, chosen).shape == (0, 12)
    dys, dweight = sp.combine_grad(none, none, chosen[:, :1], weight[:, :1], torch.zeros(5, dtype=torch.int32, device=DEV))
    assert dys.shape == (0, 12) and dweight.shape == (0, 1)


@pytest.mark.parametrize("score,normalise", SCORES)
def test_route_rows_that_masks_leave_empty(sp, score, normalise):
    inf, low = float("inf"), torch.finfo(F32).min
    logits = torch.tensor([[-inf] * 4, [float("nan")] * 4, [low] * 4, [-inf, 3.0, -inf, -inf], [low, 1.0, low, low],
                           [-200.0, -300.0, -1000.0, -90.0], [inf, 1.0, 2.0, 0.0], [80.0, 1000.0, 500.0, low]], device=DEV)
    got = sp.route(logits, 2, score=score, normalise=normalise)
    check_route(got, logits, 2, None, None, score, normalise, 1.0)
    assert got[0].tolist()[:4] == [[-1, -1], [-1, -1], [0, 1], [1, -1]]
    assert got[1][:2].abs().sum() == 0
    dw = torch.ones(8, 2, device=DEV)
    d = sp.route_grad(dw, logits, got[0], score=score, normalise=normalise)
    assert d[:2].abs().sum() == 0 and torch.isfinite(d[:6]).all()
    # an expert that the bias closes, one that it forces
    bias = torch.tensor([0.0, -inf, inf, 0.0], device=DEV)
    some = normal(1, (50, 4), F32)
    got = sp.route(some, 3, bias=bias, score=score, normalise=normalise)
    check_route(got, some, 3, bias, None, score, normalise, 1.0)
    assert (got[0][:, 0] == 2).all() and not (got[0] == 1).any()


@pytest.mark.parametrize("score,normalise", SCORES)
@pytest.mark.parametrize("rows,experts,k", [(20, 6, 3), (8, 100, 8)])
def test_route_grad_against_differences(sp, rows, experts, k, score, normalise):
    """Along a direction v of at most 1 per logit, along which no choice changes.  A softmax weight p has the third derivative
    p ((v - m)^3 - 3 (v - m) c2 - c3) with |v - m| <= 2 and cumulants c2 <= 1, c3 <= 2 of v, less than 16; under log_sigmoid,
    whose derivatives are at most 1, 1/4 and 1/8, less than 24.  Both ends are off by their rounding."""
    g = torch.Generator().manual_seed(3)
    base = torch.stack([torch.randperm(experts, generator=g) for _ in range(rows)]).float().to(DEV) * 0.125 - 1.0
    v = (torch.rand(rows, experts, generator=g) * 2 - 1).to(DEV)
    eps = 2.0 ** -7  # four times it is less than the distance of two logits
    dw = normal(4, (rows, k), F32)
    f = [sp.route(base + s * eps * v, k, score=score, normalise=normalise) for s in (1, -1)]
    chosen, _ = sp.route(base, k, score=score, normalise=normalise)
    assert torch.equal(f[0][0], chosen) and torch.equal(f[1][0], chosen)
    diff = ((f[0][1].double() - f[1][1].double()) * dw.double()).sum(1) / (2 * eps)
    d = sp.route_grad(dw, base, chosen, score=score, normalise=normalise)
    size = dw.double().abs().sum(1).cpu()
    slack = torch.from_numpy(ref.weight_slack(ref.f64(base) + eps, np.ones((rows, experts), dtype=bool), experts))[:, 0]
    off = ((d.double() * v.double()).sum(1) - diff).abs().cpu()
    assert (off <= size * (24 * eps * eps / 6 + 2 * slack / eps)).all(), (off, size)


# ---------------------------------------------------------------------------
# dispatch and back
# ---------------------------------------------------------------------------
PAIR_SIZES = [(0, 2, 4, 8), (1, 1, 1, 1), (1, 8, 256, 1024), (2, 3, 5, 7), (16, 2, 8, 64), (33, 4, 12, 777), (64, 16, 64, 65), (127, 8, 1024, 40),
              (129, 8, 100, 1500), (700, 3, 17, 33), (1030, 16, 1000, 3), (5000, 2, 3, 9), (9000, 8, 64, 2)]


def pairs(seed, rows, k, experts, dropped=True):
    rng = np.random.default_rng(seed)
    c = np.minimum(rng.geometric(min(0.9, 4 / experts), (rows, k)) - 1, experts - 1)  # uneven, repeated experts too
    if dropped:
        c[rng.random((rows, k)) < 0.1] = -1
        c[rng.random((rows, k)) < 0.03] = experts  # outside as well
        c[rows - rows // 8:] = -1
    return torch.from_numpy(c.astype(np.int32)).to(DEV)


@pytest.mark.parametrize("dropped", [False, True])
@pytest.mark.parametrize("dtype,layout", [(F32, "part"), (BF16, "dense"), (F16, "part"), (F32, "one")])
@pytest.mark.parametrize("rows,k,experts,width", PAIR_SIZES)
def test_dispatch(sp, rows, k, experts, width, dtype, layout, dropped):
    chosen = pairs(rows + k, rows, k, experts, dropped)
    x = normal(rows, (rows, width), dtype, layout)
    xs, offsets, place = sp.dispatch(x, chosen, experts)
    want_place, want_offsets = ref.sort_pairs(chosen.cpu().numpy(), experts)
    assert np.array_equal(place.cpu().numpy(), want_place)
    assert np.array_equal(offsets.cpu().numpy(), want_offsets)
    want = torch.zeros(rows * k, width, dtype=dtype)
    flat = torch.from_numpy(want_place.reshape(-1)).long()
    pair = torch.nonzero(flat >= 0)[:, 0]
    want[flat[pair]] = x.cpu()[pair // k]
    assert torch.equal(xs.cpu(), want)


@pytest.mark.parametrize("dtype,layout,weighted,add", [(F32, "part", True, True), (BF16, "dense", True, True), (BF16, "part", True, False),
                                                       (F16, "dense", False, False), (F32, "one", False, True)])
@pytest.mark.parametrize("rows,k,experts,width", PAIR_SIZES)
def test_combine(sp, rows, k, experts, width, dtype, layout, weighted, add):
    chosen = pairs(rows + k + 1, rows, k, experts)
    place = torch.from_numpy(ref.sort_pairs(chosen.cpu().numpy(), experts)[0]).to(DEV)
    ys = normal(rows + 1, (rows * k, width), dtype, layout)
    weight = normal(3, (rows, k), F32).contiguous() if weighted else None
    residual = normal(5, (rows, width), dtype, layout) if add else None
    if weighted:
        weight[place < 0] = float("nan")  # slots without an expert: not read
    if layout == "dense":
        ys[int((place >= 0).sum()):] = float("nan")
    got = sp.combine(ys, place, weight=weight, add=residual) if weighted or add else sp.dispatch_grad(ys, place)
    want, bound = ref.combine(ref.f64(ys), place.cpu().numpy(), None if weight is None else ref.f64(weight),
                              None if residual is None else ref.f64(residual))
    ref.assert_within(got, want, bound, dtype)


@pytest.mark.parametrize("dtype,layout", [(F32, "part"), (BF16, "dense"), (F16, "part"), (F32, "one")])
@pytest.mark.parametrize("rows,k,experts,width", PAIR_SIZES)
def test_combine_grad(sp, rows, k, experts, width, dtype, layout):
    chosen = pairs(rows + k + 2, rows, k, experts)
    place_np, offsets = ref.sort_pairs(chosen.cpu().numpy(), experts)
    place = torch.from_numpy(place_np).to(DEV)
    ys = normal(rows + 1, (rows * k, width), dtype, layout)
    dout = normal(rows + 2, (rows, width), dtype, layout)
    weight = normal(3, (rows, k), F32).contiguous()
    weight[place < 0] = float("nan")
    dys, dweight = sp.combine_grad(dout, ys, place, weight, torch.from_numpy(offsets).to(DEV))
    flat = torch.from_numpy(place_np.reshape(-1)).long()
    pair = torch.nonzero(flat >= 0)[:, 0]
    want = torch.zeros(rows * k, width, dtype=dtype)
    want[flat[pair]] = (weight.cpu().reshape(-1)[pair][:, None] * dout.cpu().float()[pair // k]).to(dtype)  # one product: equal
    assert torch.equal(dys.cpu(), want)
    pair, flat = pair.numpy(), flat.numpy()
    terms = ref.f64(dout)[pair // k] * ref.f64(ys)[flat[pair]]
    dw, bound = np.zeros(rows * k), np.zeros(rows * k)
    dw[pair] = terms.sum(1)
    bound[pair] = (width + 2) * ref.U * np.abs(terms).sum(1)
    ref.assert_within(dweight, dw.reshape(rows, k), bound.reshape(rows, k), F32)


def test_gradients_of_the_way_there_and_back_against_differences(sp):
    """dispatch is linear, combine bilinear: with whole numbers the differences are exact."""
    rng = np.random.default_rng(7)
    whole = lambda *shape: torch.from_numpy(rng.integers(-3, 4, shape)).float().to(DEV)
    rows, k, experts, width = 60, 3, 7, 50
    chosen = pairs(1, rows, k, experts)
    x, dx, u = whole(rows, width), whole(rows, width), whole(rows * k, width)
    xs, offsets, place = sp.dispatch(x, chosen, experts)
    moved = sp.dispatch(x + dx, chosen, experts)[0]
    assert float((u * (moved - xs)).sum()) == float((sp.dispatch_grad(u, place) * dx).sum())
    ys, dys, w, dw, dout, add = whole(rows * k, width), whole(rows * k, width), whole(rows, k), whole(rows, k), whole(rows, width), whole(rows, width)
    gys, gw = sp.combine_grad(dout, ys, place, w, offsets)
    here = sp.combine(ys, place, weight=w, add=add)
    assert float((dout * (sp.combine(ys + dys, place, weight=w, add=add) - here)).sum()) == float((gys * dys).sum())
    assert float((dout * (sp.combine(ys, place, weight=w + dw, add=add) - here)).sum()) == float((gw * dw).sum())


def test_infinities_stay_in_their_rows(sp):
    rows, k, width = 40, 2, 100
    chosen = pairs(3, rows, k, 5, dropped=False)
    x = normal(1, (rows, width), F32)
    x[7, 3], x[8] = float("inf"), float("nan")
    xs, offsets, place = sp.dispatch(x, chosen, 5)
    out = sp.combine(xs, place, weight=torch.full((rows, k), 0.5, device=DEV))
    assert torch.equal(out[:7], x[:7]) and out[7, 3] == float("inf") and torch.isfinite(out[7, 4:]).all()
    assert torch.isnan(out[8]).all() and torch.isfinite(out[9:]).all()


# ---------------------------------------------------------------------------
# streams, graphs, refusals
# ---------------------------------------------------------------------------
def mixture_step(sp, table, ids, router, k, dout):
    """Every operator once; the experts multiply by their number plus one."""
    x = sp.embed(table, ids, scale=2.0)
    logits = x[:, :router]
    chosen, weight = sp.route(logits, k)
    xs, offsets, place = sp.dispatch(x, chosen, router)
    ys = xs * 3.0
    out = sp.combine(ys, place, weight=weight, add=x)
    dys, dweight = sp.combine_grad(dout, ys, place, weight, offsets)
    dx = sp.dispatch_grad(dys, place)
    dlogits = sp.route_grad(dweight, logits, chosen)
    dtable = sp.embed_grad(dx, ids, table.shape[0])
    return chosen, weight, xs, offsets, place, out, dys, dweight, dx, dlogits, dtable


@pytest.mark.parametrize("rows", [3, 900])
def test_another_stream_and_a_graph(sp, rows):
    table, dout = normal(1, (500, 96), F32), normal(2, (rows, 96), F32)
    ids = zipf(3, rows, 500)
    want = mixture_step(sp, table, ids, 24, 4, dout)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = mixture_step(sp, table, ids, 24, 4, dout)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = mixture_step(sp, table, ids, 24, 4, dout)
    for seed in (11, 12, 13, 14):  # new contents, the same graph
        table.copy_(normal(seed, (500, 96), F32))
        ids.copy_(zipf(seed, rows, 500))
        graph.replay()
        torch.cuda.synchronize()
        want = mixture_step(sp, table, ids, 24, 4, dout)
        assert all(torch.equal(a, b) for a, b in zip(held, want)), seed


def test_refusals(sp):
    f = lambda *shape, dtype=F32: torch.zeros(*shape, dtype=dtype, device=DEV)
    i = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=DEV)
    calls = [
        lambda: sp.embed(f(4, 8, dtype=torch.float64), i(3)),
        lambda: sp.embed(f(4, 8), f(3)),
        lambda: sp.embed(f(4, 8), i(3).cpu()),
        lambda: sp.embed(f(4, 8).cpu(), i(3)),
        lambda: sp.embed(f(8, 4).t(), i(3)),
        lambda: sp.embed(f(0, 8), i(3)),
        lambda: sp.embed(f(4, 0), i(3)),
        lambda: sp.embed(f(4, 8), i(3), dtype=torch.int32),
        lambda: sp.embed_grad(f(3, 8), i(4), 10),
        lambda: sp.embed_grad(f(3, 8), i(3), 0),
        lambda: sp.embed_grad(f(3, 8), i(3), 10, out=f(9, 8)),
        lambda: sp.embed_grad(f(3, 8), i(3), 10, out=f(1, 8).expand(10, 8)),
        lambda: sp.route(f(3, 8), 0),
        lambda: sp.route(f(3, 8), -1),
        lambda: sp.route(f(3, 8), 9),
        lambda: sp.route(f(3, 40), 17),
        lambda: sp.route(f(3, 1025), 2),
        lambda: sp.route(f(3, 8), 2, bias=f(7)),
        lambda: sp.route(f(3, 8), 2, keep=f(3)),
        lambda: sp.route(f(3, 8), 2, score="tanh"),
        lambda: sp.route_grad(f(3, 2), f(3, 8), i(3, 3)),
        lambda: sp.route_grad(f(2, 3).t(), f(3, 8), i(3, 2)),
        lambda: sp.dispatch(f(3, 8), i(4, 2), 4),
        lambda: sp.dispatch(f(3, 8), i(3, 2).long(), 4),
        lambda: sp.dispatch(f(3, 8), i(3, 2), 0),
        lambda: sp.dispatch(f(3, 8), i(3, 17), 20),
        lambda: sp.dispatch(f(3, 0), i(3, 2), 4),
        lambda: sp.combine(f(5, 8), i(3, 2)),
        lambda: sp.combine(f(6, 8), i(3, 2), weight=f(2, 3)),
        lambda: sp.combine(f(6, 8), i(3, 2), add=f(3, 8, dtype=BF16)),
        lambda: sp.combine(f(6, 8), i(3, 2), add=f(3, 7)),
        lambda: sp.combine_grad(f(3, 8), f(6, 8), i(3, 2), None, i(5)),
        lambda: sp.combine_grad(f(3, 8, dtype=BF16), f(6, 8), i(3, 2), f(3, 2), i(5)),
        lambda: sp.combine_grad(f(3, 8), f(6, 8), i(3, 2), f(3, 2), i(1)),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(sp.SpdnnError) as e:
            call()
        assert e.value.code == sp.SPDNN_EINVAL, n

"""Dense products and layer norm as a program uses them: together with the row operators, on streams and in graphs, beside automatic
gradients, beyond 32 bits, and with offsets that are wrong."""
import ctypes
import warnings

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


def whole(g, shape, dtype, most=2):
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype)


# ---------------------------------------------------------------------------
# a block of a mixture: norm, router, dispatch, two products per expert, combine; and its gradients
# ---------------------------------------------------------------------------
def block(sp, p, ids, experts, k):
    x = sp.embed(p["table"], ids)
    h, stats = sp.layer_norm(x, p["gain"], p["shift"], stats=True)
    logits = sp.linear(h, p["router"], dtype=F32)
    chosen, weight = sp.route(logits, k, keep=ids >= 0)
    xs, offsets, place = sp.dispatch(h, chosen, experts)
    up, pre = sp.grouped_linear(xs, offsets, p["w1"], bias=p["b1"], act="gelu", pre=True)
    ys = sp.grouped_linear(up, offsets, p["w2"], bias=p["b2"])
    out = sp.combine(ys, place, weight=weight, add=x)
    return out, (x, h, stats, logits, chosen, weight, xs, offsets, place, up, pre, ys)


def block_grad(sp, p, ids, dout, saved):
    x, h, stats, logits, chosen, weight, xs, offsets, place, up, pre, ys = saved
    dys, dweight = sp.combine_grad(dout, ys, place, weight, offsets)
    dup, dw2, db2 = sp.grouped_linear_grad(dys, up, offsets, p["w2"])
    dxs, dw1, db1 = sp.grouped_linear_grad(dup, xs, offsets, p["w1"], pre=pre, act="gelu")
    dlogits = sp.route_grad(dweight, logits, chosen)
    dh, drouter, _ = sp.linear_grad(dlogits, h, p["router"], for_bias=False)
    dh = dh + sp.dispatch_grad(dxs, place)
    dx, dgain, dshift = sp.layer_norm_grad(dh, x, stats, p["gain"], add=dout)
    dtable = sp.embed_grad(dx, ids, p["table"].shape[0])
    return dict(table=dtable, gain=dgain, shift=dshift, router=drouter, w1=dw1, b1=db1, w2=dw2, b2=db2)


def plain_block(p, ids, chosen):
    """The same from its formulas on the CPU in 64 bits, the choice taken as given."""
    ok = ids >= 0
    x = torch.where(ok[:, None], p["table"][ids.clamp(min=0)], 0.0)
    d = x - x.mean(1, keepdim=True)
    h = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * p["gain"] + p["shift"]
    logits = h @ p["router"]
    valid = chosen >= 0
    picked = torch.where(valid, logits.gather(1, chosen.clamp(min=0)), -torch.inf)
    picked = torch.where(valid.any(1, keepdim=True), picked, 0.0)
    w = torch.where(valid, torch.softmax(picked, 1), 0.0)
    out = x
    for j in range(chosen.shape[1]):
        e = chosen[:, j].clamp(min=0)
        u = torch.einsum("ti,tio->to", h, p["w1"][e]) + p["b1"][e]
        y = torch.einsum("ti,tio->to", 0.5 * u * torch.special.erfc(-u / 2 ** 0.5), p["w2"][e]) + p["b2"][e]
        out = out + torch.where(valid[:, j:j + 1], w[:, j:j + 1] * y, 0.0)
    return out


def parameters(g, vocab, width, inner, experts):
    f = lambda *shape, scale=1.0: torch.randn(*shape, generator=g) * scale
    return dict(table=f(vocab, width), gain=1 + f(width, scale=0.1), shift=f(width, scale=0.1), router=f(width, experts, scale=width ** -0.5),
                w1=f(experts, width, inner, scale=width ** -0.5), b1=f(experts, inner, scale=0.1), w2=f(experts, inner, width, scale=inner ** -0.5),
                b2=f(experts, width, scale=0.1))


def test_a_block_of_a_mixture(sp):
    g = torch.Generator().manual_seed(3)
    n, vocab, width, inner, experts, k = 90, 40, 72, 100, 6, 2
    p = parameters(g, vocab, width, inner, experts)
    ids = torch.randint(0, vocab, (n,), generator=g)
    ids[-9:] = -1
    dout = torch.randn(n, width, generator=g)
    dev = {name: t.to(DEV) for name, t in p.items()}
    dev["w2"] = p["w2"].transpose(1, 2).contiguous().to(DEV).transpose(1, 2)  # stored the other way round
    out, saved = block(sp, dev, ids.to(DEV), experts, k)
    grads = block_grad(sp, dev, ids.to(DEV), dout.to(DEV), saved)
    leaves = {name: t.double().requires_grad_() for name, t in p.items()}
    chosen = saved[4].cpu().long()
    want = plain_block(leaves, ids, chosen)
    want.backward(dout.double())
    # Five steps of at most a few hundred 32-bit additions each, U of the largest terms apart, amplified by rstd (below 1.5 here): a
    # thousand times U of the largest number is beyond all of it.
    U = 2.0 ** -24
    assert float((out.cpu().double() - want.detach()).abs().max()) <= 1000 * U * float(want.detach().abs().max())
    for name, t in leaves.items():
        off = float((grads[name].cpu().double() - t.grad).abs().max())
        assert off <= 1000 * U * float(t.grad.abs().max()), (name, off, float(t.grad.abs().max()))
    # token by token: the same
    for t in (0, 5, n - 1):
        one, _ = block(sp, dev, ids[t:t + 1].to(DEV), experts, k)
        assert float((one.cpu() - out[t:t + 1].cpu()).abs().max()) <= 1000 * U * float(want.detach().abs().max())


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_a_block_in_a_graph(sp, dtype):
    """Forward and gradients captured, replayed with new tokens between eager calls of the same; two graphs that run in turn."""
    g = torch.Generator().manual_seed(4)
    n, vocab, width, inner, experts, k = 200, 50, 136, 264, 5, 2
    p = {name: t.to(dtype).to(DEV) for name, t in parameters(g, vocab, width, inner, experts).items()}
    ids = torch.randint(0, vocab, (n,), generator=g).to(DEV)
    dout = torch.randn(n, width, generator=g).to(dtype).to(DEV)

    def step():
        out, saved = block(sp, p, ids, experts, k)
        return [out] + list(block_grad(sp, p, ids, dout, saved).values())

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        graphs.append((graph, captured))
    for turn in range(4):
        ids.copy_(torch.randint(-1, vocab, (n,), generator=g))
        graph, captured = graphs[turn % 2]
        graph.replay()
        again = [t.clone() for t in captured]
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(again, eager):
            assert torch.equal(a, b), turn


def test_results_do_not_depend_on_timing(sp):
    """Sums in parts and by several waves give the same bits every time, beside other work and on other streams."""
    g = torch.Generator().manual_seed(5)
    x, w, d = torch.randn(900, 2000, generator=g).to(DEV), torch.randn(2000, 70, generator=g).to(DEV), torch.randn(900, 70, generator=g).to(DEV)
    big = torch.randn(4096, 4096, device=DEV)
    first = [sp.linear(x, w), sp.linear(x[:3], w), *sp.linear_grad(d, x, w), *sp.layer_norm_grad(x, x, sp.layer_norm(x, stats=True)[1])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for turn in range(5):
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            if turn % 3:
                big @ big
            again = [sp.linear(x, w), sp.linear(x[:3], w), *sp.linear_grad(d, x, w), *sp.layer_norm_grad(x, x, sp.layer_norm(x, stats=True)[1])]
        torch.cuda.synchronize()
        for a, b in zip(first, again):
            assert torch.equal(a, b), turn


def test_rows_and_weights_beyond_32_bits(sp):
    g = torch.Generator().manual_seed(6)
    # rows of x beyond 2^32 bytes, and a stride that no tile of 32-bit offsets reaches
    rows, stride = 40000, 65600
    big = torch.empty(rows * stride, dtype=BF16, device=DEV)
    x = big.view(rows, stride)[:, 3:67]
    few = torch.tensor([0, 1, 12345, rows - 2, rows - 1])
    x.zero_()
    x[few] = whole(g, (5, 64), BF16).to(DEV)
    w = whole(g, (64, 96), BF16).to(DEV)
    out = sp.linear(x, w)
    assert torch.equal(out[few], (x[few].double() @ w.double()).to(BF16)) and not out[2:12345].any()
    d = torch.zeros(rows, 96, dtype=BF16, device=DEV)
    d[few] = whole(g, (5, 96), BF16).to(DEV)
    dx, dw, db = sp.linear_grad(d, x, w, dtype=F32)
    assert torch.equal(dw.double(), x[few].double().t() @ d[few].double()) and torch.equal(db.double(), d[few].double().sum(0))
    assert torch.equal(dx[few], (d[few].double() @ w.double().t()).to(BF16))
    far = big[:300 * 5000000].view(300, 5000000)[:, 1:65]
    far.copy_(whole(g, (300, 64), BF16))
    assert torch.equal(sp.linear(far, w), (far.double() @ w.double()).to(BF16))
    assert torch.equal(sp.layer_norm(far), sp.layer_norm(far.contiguous()))
    # outputs beyond 2^32 elements
    wide = whole(g, (64, 110000), BF16).to(DEV)
    out = sp.linear(x, wide)
    assert out.numel() > 2 ** 32
    assert torch.equal(out[few[-2:]], (x[few[-2:]].double() @ wide.double()).to(BF16))
    del out, far, x, big
    # experts' weights beyond 2^32 bytes
    experts, width, cols = 160, 4096, 4096
    we = torch.empty(experts, width, cols, dtype=BF16, device=DEV)
    we[experts - 1] = whole(g, (width, cols), BF16, 1).to(DEV)
    we[0] = whole(g, (width, cols), BF16, 1).to(DEV)
    xs = whole(g, (300, width), BF16, 1).to(DEV)
    offsets = torch.zeros(experts + 1, dtype=torch.int32)
    offsets[1:] = 150
    offsets[experts] = 300
    for w in (we, we.transpose(1, 2)):
        out = sp.grouped_linear(xs, offsets.to(DEV), w, dtype=F32)
        assert torch.equal(out[:150].double(), xs[:150].double() @ w[0].double())
        assert torch.equal(out[150:].double(), xs[150:].double() @ w[experts - 1].double())
        dw = sp.grouped_linear_grad(xs, xs, offsets.to(DEV), w, for_x=False, for_bias=False)[1]
        assert torch.equal(dw[experts - 1].double(), (xs[150:].double().t() @ xs[150:].double()).to(BF16).double()) and not dw[1:-1].any()
        del out, dw


@pytest.mark.parametrize("rows,width,cols", [(200, 32, 48), (40, 64, 80), (900, 64, 300)])
def test_wrong_offsets_touch_nothing_else(sp, rows, width, cols):
    """Offsets that do not ascend within 0 .. rows: the rows are not specified, and what lies around the outputs stays."""
    L, n = sp.lib(), 4
    x, w = torch.ones(rows, width, device=DEV), torch.ones(n, width, cols, device=DEV)
    size = ctypes.c_size_t()
    assert L.spdnn_linear_bytes(rows, width, cols, 1, n, 0, ctypes.byref(size)) == 0
    need = size.value
    assert L.spdnn_linear_grad_bytes(rows, width, cols, 1, n, 0, 0, 0, 0, ctypes.byref(size)) == 0
    need = max(need, size.value)
    room = 4096

    def guarded(count):
        t = torch.full((count + 2 * room,), 5.0, device=DEV)
        return t, t.data_ptr() + 4 * room

    for at in ([0, 300, 50, 900, 200], [-5, -9, 2 ** 31 - 1, -2 ** 31, 7], [200, 150, 100, 50, 0], [7, 7, 7, 7, 7], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        off = torch.tensor(at, dtype=torch.int32, device=DEV)
        out, outp = guarded(rows * cols)
        dx, dxp = guarded(rows * width)
        dw, dwp = guarded(n * width * cols)
        db, dbp = guarded(n * cols)
        work, workp = guarded(need // 4)
        workp -= workp % 256
        stream = torch.cuda.current_stream().cuda_stream
        assert L.spdnn_linear(x.data_ptr(), 0, rows, width, width, off.data_ptr(), n, w.data_ptr(), 0, cols, width * cols, cols, 0, 0, 0, 0, cols, outp, 0,
                              cols, 0, cols, workp, need, stream) == 0
        assert L.spdnn_linear_grad(outp, 0, cols, 0, cols, 0, x.data_ptr(), 0, rows, width, width, off.data_ptr(), n, w.data_ptr(), 0, cols, width * cols, cols,
                                   dxp, width, dwp, cols, width * cols, dbp, 0, workp, need, stream) == 0
        torch.cuda.synchronize()
        for t in (out, dx, dw, db, work):
            edge = room - 64  # work begins at a multiple of 256 bytes, up to 64 floats before
            assert bool((t[:edge] == 5).all()) and bool((t[-edge:] == 5).all()), at


def inputs(dtype=F32):
    g = torch.Generator().manual_seed(1)
    f = lambda *shape: torch.randn(*shape, generator=g).to(dtype).to(DEV)
    return dict(x=f(6, 8), w=f(8, 5), we=f(2, 8, 5), b=f(5), be=f(2, 5), add=f(6, 5), dout=f(6, 5), pre=f(6, 5), n=f(8), dn=f(6, 8), stats=torch.rand(6, 2, device=DEV),
                off=torch.tensor([0, 4, 6], dtype=torch.int32, device=DEV))


CALLS = [
    ("linear", lambda sp, t: sp.linear(t["x"], t["w"], bias=t["b"], add=t["add"]), ["x", "w", "b", "add"]),
    ("grouped_linear", lambda sp, t: sp.grouped_linear(t["x"], t["off"], t["we"], bias=t["be"], add=t["add"]), ["x", "we", "be", "add"]),
    ("linear_grad", lambda sp, t: sp.linear_grad(t["dout"], t["x"], t["w"], pre=t["pre"], act="silu"), ["dout", "x", "w", "pre"]),
    ("grouped_linear_grad", lambda sp, t: sp.grouped_linear_grad(t["dout"], t["x"], t["off"], t["we"], pre=t["pre"], act="silu"), ["dout", "x", "we", "pre"]),
    ("layer_norm", lambda sp, t: sp.layer_norm(t["x"], t["n"], t["n"]), ["x", "n"]),
    ("layer_norm_grad", lambda sp, t: sp.layer_norm_grad(t["dn"], t["x"], t["stats"], t["n"], add=t["dn"]), ["dn", "x", "n"]),
]


@pytest.mark.parametrize("name,call,leaves", CALLS, ids=[c[0] for c in CALLS])
def test_a_call_warns_where_a_gradient_would_be_lost(sp, name, call, leaves):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        call(sp, inputs())
        for leaf in leaves:
            t = inputs()
            t[leaf].requires_grad_()
            with torch.no_grad():
                call(sp, t)
            with pytest.raises(UserWarning, match="^%s records no gradient" % name):
                call(sp, t)


def test_the_warning_names_the_caller(sp):
    for _, call, leaves in CALLS:
        t = inputs()
        t[leaves[0]].requires_grad_()
        with warnings.catch_warnings(record=True) as seen:
            warnings.simplefilter("always")
            call(sp, t)
        assert len(seen) == 1 and seen[0].filename == __file__


def test_what_is_refused(sp):
    t = inputs()
    host = torch.zeros(6, 8)
    for call in (lambda: sp.linear(host, t["w"]), lambda: sp.linear(t["x"], t["w"].cpu()), lambda: sp.linear(t["x"], t["w"], bias=t["b"].cpu()),
                 lambda: sp.linear(t["x"].t(), t["w"]), lambda: sp.grouped_linear(t["x"], t["off"].cpu(), t["we"]),
                 lambda: sp.grouped_linear(t["x"], t["off"].long(), t["we"]), lambda: sp.linear_grad(t["dout"], t["x"], t["w"], act="gelu"),
                 lambda: sp.layer_norm(host), lambda: sp.layer_norm_grad(t["dn"], t["x"], t["stats"].half())):
        with pytest.raises(sp.SpdnnError):
            call()

"""The activations of the dense products over their whole range: negative arguments far out, where little is left of the result, and
infinities.  Arguments reach them exactly, as products with ones, and slopes leave them as products with the identity."""
import math

import pytest
import torch

import dense_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = ref.TYPES
U = ref.U
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def activated(sp, x, act, cols):
    """act(x) by way of many rows, and by way of one row with many columns."""
    ones = torch.ones(1, cols, dtype=x.dtype, device=DEV)
    many = sp.linear(x.to(DEV).view(-1, 1), ones, act=act)
    one = sp.linear(torch.ones(1, 1, dtype=x.dtype, device=DEV), x.to(DEV).view(1, -1), act=act)
    return [many[:, 0].cpu(), many[:, cols - 1].cpu(), one[0].cpu()]


def slopes(sp, pre, act, cols):
    """act'(pre), with dout of ones."""
    dout, eye = torch.ones(len(pre), cols, dtype=pre.dtype, device=DEV), torch.eye(cols, dtype=pre.dtype, device=DEV)
    dx = sp.linear_grad(dout, dout, eye, pre=pre.to(DEV).view(-1, 1).repeat(1, cols), act=act, for_weight=False, for_bias=False)[0]
    return [dx[:, 0].cpu(), dx[:, cols - 1].cpu()]


def arguments(dtype, least, most):
    x = torch.cat([torch.linspace(least, most, 3001), torch.tensor([-1e-3, -2.0 ** -20, 0.0, 2.0 ** -20])])
    return x.to(dtype).unique()


# Relative errors.  16 bits: the tail's polynomial is off by 6e-5; its argument by 4 U, to which it answers at most threefold; six steps
# by 2 U of terms whose magnitudes add up to three times the result at most: 48 U in all.  exp2 is off by 2 U, its argument by three
# roundings of x^2 / 2 and one of the factor: 2 U x^2.  Floats: the product with 1 / sqrt 2 is off by 2 U, to which erfc answers (x^2 + 1)-fold;
# erfcf by 8 U (4 ulp), products and the sum by 4 U.  exp(-x^2 / 2) of the slope: two roundings of its argument, 8 U else.
def tail_off(x, dtype):
    return (2 * x * x + 16) * U if dtype == F32 else 6e-5 + (2 * x * x + 52) * U


def bell_off(x, dtype):
    return (2 * x * x + 12) * U


@pytest.mark.parametrize("cols", [1, 8, 11])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_gelu_keeps_its_digits(sp, dtype, cols):
    """gelu(x) = x Phi(x) relative to itself for negative x."""
    x = arguments(dtype, -12.0, 12.0)
    z = x.double()
    tail = 0.5 * torch.special.erfc(z.abs() / math.sqrt(2))
    want = z.clamp(min=0) - z.abs() * tail
    off = z.abs() * tail * tail_off(z, dtype) + U * want.abs()
    for got in activated(sp, x, "gelu", cols):
        ref.assert_within(got, want.numpy(), off.numpy(), dtype, "gelu")


@pytest.mark.parametrize("cols", [1, 8, 11])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_the_slope_of_gelu_keeps_its_digits(sp, dtype, cols):
    """Phi(x) + x phi(x), each relative to itself for negative x."""
    x = arguments(dtype, -12.0, 12.0)
    z = x.double()
    tail = 0.5 * torch.special.erfc(z.abs() / math.sqrt(2))
    bell = z.abs() * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    want = torch.where(z < 0, tail - bell, 1 - (tail - bell))
    off = tail * tail_off(z, dtype) + bell * bell_off(z, dtype) + U * ((tail - bell).abs() + (z >= 0) * want.abs())
    for got in slopes(sp, x, "gelu", cols):
        ref.assert_within(got, want.numpy(), off.numpy(), dtype, "slope")


# sigmoids: exp is off by 4 U, its argument by 2 U |x| (16 bits: a product and its factor); sum, quotient and products by 6 U.
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_silu_keeps_its_digits(sp, dtype):
    """x / (1 + exp(-x)) and its slope relative to their terms, down to where exp(x) leaves the normal numbers of 32 bits (and silu becomes 0)."""
    x = arguments(dtype, -87.0, 87.0)
    z = x.double()
    s, o = torch.sigmoid(z), torch.sigmoid(-z)
    rel = (2 * z.abs() + 10) * U
    for got in activated(sp, x, "silu", 9):
        ref.assert_within(got, (z * s).numpy(), ((z * s).abs() * rel).numpy(), dtype, "silu")
    for got in slopes(sp, x, "silu", 9):
        ref.assert_within(got, (s * (1 + z * o)).numpy(), (s * rel + 2 * (z * s * o).abs() * rel + 4 * U * s).numpy(), dtype, "slope")


def ends(dtype):
    big = {F32: 1e38, BF16: 1e38, F16: 65504.0}[dtype]
    return torch.tensor([-INF, -big, -100.0, 100.0, big, INF, NAN], dtype=dtype)


ENDS = ["gelu", "silu"]


@pytest.mark.parametrize("act", ENDS)
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_the_ends_of_activations(sp, dtype, act):
    """0 and x at the infinities, slopes 0 and 1; a NaN stays one."""
    x = ends(dtype)
    for cols in (1, 8):
        for got in activated(sp, x, act, cols):
            assert not got[:3].abs().gt(1e-37).any() and torch.equal(got[3:6], x[3:6]) and got[6].isnan(), got
        for got in slopes(sp, x, act, cols):
            assert not got[:3].abs().gt(1e-37).any() and torch.equal(got[3:6], torch.ones(3, dtype=dtype)) and got[6].isnan(), got


@pytest.mark.parametrize("act", ENDS)
def test_gradients_where_pre_leaves_16_bits(sp, act):
    """A sum of -90000 is -inf in float16: out is 0, and so are the gradients."""
    x, w = torch.full((5, 300), -1.0, dtype=F16, device=DEV), torch.full((300, 24), 300.0, dtype=F16, device=DEV)
    out, pre = sp.linear(x, w, act=act, pre=True)
    assert not out.any() and bool((pre == -INF).all())
    for grad in sp.linear_grad(torch.ones_like(out), x, w, pre=pre, act=act):
        assert not grad.any()


# one column to several workgroups of 512, one row to several chunks; experts that begin within a chunk, with one row and with none
SUMS = [(1, 1, None), (3, 9, None), (17, 40, None), (1000, 513, None), (5000, 1100, None), (40, 24, [0, 1, 1, 2, 16, 17, 33, 40]), (700, 30, [0, 0, 700]),
        (900, 520, [0, 100, 100, 101, 640, 880]), (2000, 16, list(range(0, 1001)) + [1999])]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype,wide,act", [(BF16, False, "gelu"), (BF16, True, None), (F16, True, "silu"), (F16, False, "clip"), (F32, False, "gelu")])
@pytest.mark.parametrize("rows,cols,at", SUMS, ids=lambda v: "-".join(map(str, v[:7])) if isinstance(v, list) else str(v))
def test_dbias_is_a_sum_of_32_bits(sp, rows, cols, at, dtype, wide, act, transposed):
    """dbias sums dout * act'(pre) as it is before it is rounded to 16 bits for the products."""
    g = torch.Generator().manual_seed(rows + cols)
    width, sets = 24, () if at is None else (len(at) - 1,)
    kind = F32 if wide else dtype
    x, dout, pre = torch.randn(rows, width, generator=g).to(dtype), torch.randn(rows, cols, generator=g).to(kind), (2 * torch.randn(rows, cols, generator=g)).to(kind)
    w = torch.randn(sets + ((cols, width) if transposed else (width, cols)), generator=g).to(dtype)
    d, z = dout.double(), pre.double()
    s = ref.slope(z, act)
    d, off = d * s, d.abs() * ref.slope_off(z, act) + U * (d * s).abs()
    want, room = [], []
    for a, b in [(0, rows)] if at is None else list(zip(at, at[1:])):
        want.append(d[a:b].sum(0))
        room.append(off[a:b].sum(0) + 2 * (b - a + 1) * U * (d[a:b].abs() + off[a:b]).sum(0))
    if at is not None:
        dout[at[-1]:], pre[at[-1]:] = NAN, NAN
    want, room = torch.stack(want).view(sets + (cols,)), torch.stack(room).view(sets + (cols,))
    w = w.to(DEV).transpose(-1, -2) if transposed else w.to(DEV)
    args = (dout.to(DEV), x.to(DEV)) + (() if at is None else (torch.tensor(at, dtype=torch.int32, device=DEV),)) + (w,)
    call = sp.linear_grad if at is None else sp.grouped_linear_grad
    every = call(*args, pre=pre.to(DEV), act=act, dtype=F32)
    ref.assert_within(every[2], want.numpy(), room.numpy(), F32, "dbias")
    assert torch.equal(call(*args, pre=pre.to(DEV), act=act, dtype=F32, for_x=False, for_weight=False)[2], every[2]) or dtype == F32
    ref.assert_within(call(*args, pre=pre.to(DEV), act=act, dtype=dtype, for_x=False)[2], want.numpy(), room.numpy(), dtype, "dbias of x's type")


def test_dbias_of_numbers_beyond_16_bits(sp):
    """A dout of floats that float16 does not hold."""
    dout = torch.full((40, 16), 1e5, device=DEV)
    db = sp.linear_grad(dout, torch.ones(40, 8, dtype=F16, device=DEV), torch.ones(8, 16, dtype=F16, device=DEV), dtype=F32, for_x=False, for_weight=False)[2]
    assert torch.equal(db.cpu(), torch.full((16,), 4e6))


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_weights_of_one_row(sp, dtype):
    """A row whose columns lie apart, and one number for all columns."""
    g = torch.Generator().manual_seed(1)
    x, w = torch.randint(-3, 4, (70, 1), generator=g).to(dtype), torch.randint(-3, 4, (6, 130, 5), generator=g).to(dtype)
    for weight in (w.to(DEV)[:1, :, 2], w.to(DEV)[:1, :1, 2].expand(1, 130)):
        want = x.double() @ weight.cpu().double()
        assert torch.equal(sp.linear(x.to(DEV), weight).cpu().double(), want)
        dx, dw, db = sp.linear_grad(want.to(dtype).to(DEV), x.to(DEV), weight, dtype=F32)
        assert torch.equal(dw.cpu().double(), x.double().t() @ want) and torch.equal(dx.cpu(), (want @ weight.cpu().double().t()).to(dtype))

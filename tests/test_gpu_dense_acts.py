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

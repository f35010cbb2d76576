"""The router's weights and their gradient where the bounds of its arithmetic are tightest."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, TINY = ref.U, ref.SMALLEST[torch.float32]


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


@pytest.mark.parametrize("rows,experts", [(1, 4), (50, 8), (33, 40), (9, 200), (5, 600), (4, 1024)])
def test_softmax_of_logits_that_are_exact(sp, rows, experts):
    """Softmax over all with the largest logit 0 and the others down to the smallest subnormal float's logarithm.  The difference to
    the largest is exact then, so no error grows with the logits: exp is off by 4 U (2 ulp), the sum by experts U on top,
    a quotient and a product by 2 U.  A weight is the quotient of the two; a gradient has a weight, one more quotient, exp and
    three products, and subnormal numbers are off by one of them in each of the three steps that make one."""
    g = torch.Generator().manual_seed(rows + experts)
    logits = -0.5 - 102.5 * torch.rand(rows, experts, generator=g)
    logits[torch.arange(rows), torch.randint(0, experts, (rows,), generator=g)] = 0.0
    k = min(experts, 16)
    l = ref.f64(logits)
    p = np.exp(l) / np.exp(l).sum(1, keepdims=True)
    chosen, weight = sp.route(logits.to(DEV), k, normalise=False)
    want, _ = ref.choose(logits.numpy(), k)
    assert np.array_equal(chosen.cpu().numpy(), want)
    picked = np.take_along_axis(p, want, 1)
    ref.assert_within(weight, picked, (experts + 10) * U * picked + 3 * TINY, torch.float32)
    # one expert: d = p_e (1 - p_e) for it, -p_i p_e for the others
    first = chosen[:, :1].contiguous()
    got = sp.route_grad(torch.ones(rows, 1, device=DEV), logits.to(DEV), first, normalise=False)
    pe = picked[:, :1]
    d = -p * pe
    np.put_along_axis(d, want[:, :1], pe * (1 - pe), 1)
    ref.assert_within(got, d, (2 * experts + 24) * U * p * (1 + pe) + 3 * TINY, torch.float32)


SCORES = [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)]


def check(sp, rows, experts, k, dtype, layout, with_bias, masked, score, normalise):
    """route and route_grad against the reference whose bounds the masked logits do not widen."""
    logits, bias, keep = ref.router_input(rows + experts + k, rows, experts, dtype, with_bias, masked)
    on = logits.to(DEV)
    if layout == "part":  # rows of a wider matrix, off by one element
        on = torch.cat([on[:, :1], on, on[:, :2]], 1)[:, 1:experts + 1]
    b = None if bias is None else bias.to(DEV)
    chosen, is_open = ref.choose_all(logits, k, bias, keep)
    dw = torch.randn(rows, k, generator=torch.Generator().manual_seed(k))
    dw[torch.from_numpy(chosen < 0)] = float("nan")  # not used
    l = np.where(is_open, ref.f64(logits), -np.inf)
    w, wbound, d, dbound = ref.router(l, is_open, chosen, score, normalise, 2.5, ref.f64(dw))
    got = sp.route(on, k, bias=b, keep=None if keep is None else keep.to(DEV), score=score, normalise=normalise, scale=2.5)
    assert np.array_equal(got[0].cpu().numpy(), chosen)
    ref.assert_within(got[1], w, wbound, torch.float32)
    grad = sp.route_grad(dw.to(DEV), on, got[0], bias=b, score=score, normalise=normalise, scale=2.5)
    ref.assert_within(grad, d, dbound, dtype)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,layout,with_bias", [(torch.float32, "dense", False), (torch.bfloat16, "part", True), (torch.float16, "dense", True)])
@pytest.mark.parametrize("score,normalise", SCORES)
@pytest.mark.parametrize("rows,experts,k", [(1, 1, 1), (5, 3, 2), (64, 8, 2), (3, 16, 16), (33, 63, 4), (40, 100, 16), (130, 128, 1), (31, 256, 8),
                                            (20, 257, 16), (27, 1000, 5), (14, 1024, 16)])
def test_weights_and_gradient_of_masked_rows(sp, rows, experts, k, score, normalise, dtype, layout, with_bias, masked):
    check(sp, rows, experts, k, dtype, layout, with_bias, masked, score, normalise)


@pytest.mark.parametrize("dtype,layout,with_bias,masked", [(torch.float32, "dense", False, False), (torch.float32, "part", True, True),
                                                           (torch.bfloat16, "part", True, True), (torch.float16, "dense", False, True)])
@pytest.mark.parametrize("score,normalise", SCORES)
@pytest.mark.parametrize("rows,experts,k", [(4096, 256, 8), (4097, 256, 8), (4101, 1000, 5), (4099, 257, 16), (4098, 1024, 16), (4099, 400, 1),
                                            (9001, 65, 2), (60000, 64, 4)])
def test_many_rows(sp, rows, experts, k, score, normalise, dtype, layout, with_bias, masked):
    """More rows than get a lane for every eight logits: teams of 8 and 16 lanes, which take a long row in turns."""
    check(sp, rows, experts, k, dtype, layout, with_bias, masked, score, normalise)


@pytest.mark.parametrize("rows,experts,k", [(4097, 300, 8), (4101, 1024, 16)])
def test_many_rows_take_the_first_of_equals(sp, rows, experts, k):
    few = torch.randint(-2, 3, (rows, experts), generator=torch.Generator().manual_seed(rows)).float()
    few[1] = 0.0
    few[1, ::2] = -0.0  # equal to 0
    few[2] = -float("inf")
    few[3, 7:] = float("nan")
    want, _ = ref.choose_all(few, k)
    assert want[1].tolist() == list(range(k)) and (want[2] == -1).all()
    assert np.array_equal(sp.route(few.to(DEV), k)[0].cpu().numpy(), want)

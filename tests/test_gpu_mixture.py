"""examples/sparse_mixture.py: what it gives, token by token and for a batch, and its gradients against automatic ones of the
same formulas in 64 bits."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mixture():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import sparse_mixture
    m = sparse_mixture.Mixture(300, N=256, L=2, experts=6, k=2)
    yield m
    m.close()


def dense(m, ids, saved, leaves):
    """The mixture's formulas in 64 bits; the networks' outputs and the choice are those of the forward pass."""
    table, router, gain = leaves
    _, _, _, chosen, _, xs, offsets, place, ys, expert, skip = saved
    used = len(expert)
    net = torch.zeros_like(ys)
    net[:used] = ys[:used] - skip * xs[:used]
    net = net.double()
    x = table[ids.clamp(min=0).long()] * (ids >= 0)[:, None]
    p = torch.softmax((x @ router).gather(1, chosen.clamp(min=0).long()), 1)
    out = x
    for j in range(m.k):
        there = (place[:, j] >= 0)[:, None]
        y = net[place[:, j].clamp(min=0).long()] + gain[chosen[:, j].clamp(min=0).long()] * x
        out = out + torch.where(there, p[:, j:j + 1] * y, 0.0)
    return out


@pytest.mark.parametrize("n", [1, 7, 600])
def test_mixture_and_its_gradients(mixture, n):
    print("mixture", n, flush=True)
    m = mixture
    ids = torch.randint(0, 300, (n,), generator=torch.Generator().manual_seed(n)).cuda()
    if n > 1:
        ids[-n // 5:] = -1
    out, saved = m.forward(ids)
    leaves = [t.double().requires_grad_() for t in (m.table, m.router, m.gain)]
    want = dense(m, ids, saved, leaves)
    # float32 products with inner lengths of up to 256: a few hundred roundings of values that are as large as these
    size = float(want.detach().abs().max())
    assert float((out.double() - want.detach()).abs().max()) < 300 * 2.0 ** -24 * size
    dout = torch.randn(out.shape, generator=torch.Generator().manual_seed(n + 1)).cuda()
    want.backward(dout.double())
    for got, leaf in zip(m.gradients(dout, saved), leaves):
        assert float((got.double() - leaf.grad).abs().max()) <= 600 * 2.0 ** -24 * max(float(leaf.grad.abs().max()), size)


def test_one_token_at_a_time(mixture):
    ids = torch.tensor([5, 299, -1, 5, 17], device="cuda:0")
    whole, _ = mixture.forward(ids)
    assert not whole[2].any()
    for t in range(5):
        # the product with the router may be summed in another order for one row
        one = mixture.forward(ids[t:t + 1])[0][0]
        assert float((one - whole[t]).abs().max()) <= 1e-4 * max(1.0, float(whole[t].abs().max()))

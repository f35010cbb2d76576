"""The row operators beside automatic gradients: they record nothing, say so where that would lose a gradient, and what they write
in place counts as changed."""
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def sp():
    import paper_2007_14152_amd as package
    return package


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def test_a_gradient_added_in_place_counts_as_a_change(sp):
    dout, ids = torch.ones(3, 8, device=DEV), torch.tensor([1, 2, 1], device=DEV)
    out = torch.zeros(5, 8, device=DEV)
    before = out._version
    sp.embed_grad(dout, ids, 5)
    assert out._version == before
    sp.embed_grad(dout, ids, 5, out=out)
    assert out._version > before
    # what an automatic gradient has kept is then refused, as after any other change in place
    leaf = torch.ones(8, device=DEV, requires_grad=True)
    kept = torch.ones(5, 8, device=DEV)
    loss = (leaf * kept).sum()
    sp.embed_grad(dout, ids, 5, out=kept)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        sp.embed_grad(dout, ids, 5, out=torch.zeros(5, 8, device=DEV))


def inputs():
    g = torch.Generator().manual_seed(1)
    f = lambda *shape: torch.randn(*shape, generator=g).to(DEV)
    place = torch.tensor([[0, 2], [3, -1], [1, 4]], dtype=torch.int32, device=DEV)
    return dict(table=f(9, 8), ids=torch.tensor([1, -1, 4], device=DEV), x=f(3, 8), logits=f(3, 5), bias=f(5), ys=f(6, 8), weight=f(3, 2), add=f(3, 8),
                dout=f(3, 8), dweight=f(3, 2), out=f(9, 8), place=place, chosen=torch.tensor([[0, 1], [1, -1], [0, 4]], dtype=torch.int32, device=DEV),
                offsets=torch.tensor([0, 2, 4, 4, 4, 5], dtype=torch.int32, device=DEV))


# every call with its inputs that may ask for a gradient
CALLS = [
    ("embed", lambda sp, t: sp.embed(t["table"], t["ids"]), ["table"]),
    ("embed_grad", lambda sp, t: sp.embed_grad(t["dout"], t["ids"], 9), ["dout"]),
    ("embed_grad", lambda sp, t: sp.embed_grad(t["dout"], t["ids"], 9, out=t["out"]), ["dout", "out"]),
    ("route", lambda sp, t: sp.route(t["logits"], 2, bias=t["bias"]), ["logits", "bias"]),
    ("route_grad", lambda sp, t: sp.route_grad(t["dweight"], t["logits"], t["chosen"], bias=t["bias"]), ["dweight", "logits", "bias"]),
    ("dispatch", lambda sp, t: sp.dispatch(t["x"], t["chosen"], 5), ["x"]),
    ("dispatch_grad", lambda sp, t: sp.dispatch_grad(t["ys"], t["place"]), ["ys"]),
    ("combine", lambda sp, t: sp.combine(t["ys"], t["place"], weight=t["weight"], add=t["add"]), ["ys", "weight", "add"]),
    ("combine_grad", lambda sp, t: sp.combine_grad(t["dout"], t["ys"], t["place"], t["weight"], t["offsets"]), ["dout", "ys", "weight"]),
]


def both(result):
    return result if isinstance(result, tuple) else (result,)


@pytest.mark.parametrize("name,call,wanted", CALLS)
def test_a_gradient_that_would_be_lost_is_said(sp, name, call, wanted):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        want = [r.clone() for r in both(call(sp, inputs()))]
    for which in wanted:
        t = inputs()
        t[which].requires_grad_()
        with pytest.warns(UserWarning, match="%s records no gradient" % name) as said:
            got = both(call(sp, t))
        assert [w.filename for w in said] == [__file__]  # the caller's line
        assert all(torch.equal(a, b) for a, b in zip(got, want))  # and the same results
        with warnings.catch_warnings(), torch.no_grad():
            warnings.simplefilter("error")
            t = inputs()
            t[which].requires_grad_()
            call(sp, t)

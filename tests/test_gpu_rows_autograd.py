"""The row operators beside automatic gradients: what they write in place counts as changed."""
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

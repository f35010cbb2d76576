"""The sizes that the GPU tests of the dense products run come to every kernel and tile there is, so that no change of the rule that chooses
them leaves one without a test."""
import pytest

import dense_plans as plans

TILES_16 = {"64.2", "64.3", "128.2", "128.3", "256"}
TILES_32 = {"64.2", "128.2", "256"}
# (k in parts never pays with tiles of 256 in floats, nor of 128 where one workgroup a CU is all there is)
PARTS_16 = {"64.2/s", "64.3/s", "128.2/s", "256/s"}
PARTS_32 = {"64.2/s", "128.2/s"}


@pytest.mark.parametrize("float32", [False, True])
@pytest.mark.parametrize("k_adjacent", [False, True])
def test_products(float32, k_adjacent):
    one, grouped = (plans.PRODUCTS_32, plans.GROUPED_32) if float32 else (plans.PRODUCTS_16, plans.GROUPED_16)
    for name, rows, k, cols in one:
        assert plans.product(rows, k, cols, None, float32, k_adjacent) == name, (rows, k, cols)
    for name, loads, dropped, k, cols in grouped:
        assert plans.product(sum(loads) + dropped, k, cols, len(loads), float32, k_adjacent) == name, (loads, k, cols)
    every = (TILES_32 | PARTS_32) if float32 else (TILES_16 | PARTS_16)
    assert every <= {p[0] for p in one} and every <= {p[0] for p in grouped}


@pytest.mark.parametrize("float32", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
def test_gradients_of_w(float32, transposed):
    one, grouped = (plans.GRADS_32, plans.GROUPED_GRADS_32) if float32 else (plans.GRADS_16, plans.GROUPED_GRADS_16)
    for name, rows, width, cols in one:
        assert plans.weight_grad(rows, *((cols, width) if transposed else (width, cols)), None, float32) == name, (rows, width, cols)
    for name, loads, dropped, width, cols in grouped:
        assert plans.weight_grad(sum(loads) + dropped, *((cols, width) if transposed else (width, cols)), len(loads), float32) == name, (loads, width, cols)
    assert (TILES_32 | PARTS_32) <= {p[0] for p in one} if float32 else (TILES_16 | PARTS_16) <= {p[0] for p in one}
    # (experts' own k is short: parts of it with larger tiles, and three stages of tiles of 128, come up for no sizes that were found)
    assert (TILES_32 | PARTS_32 if float32 else TILES_16 - {"128.3"} | {"64.2/s", "64.3/s"}) <= {p[0] for p in grouped}


@pytest.mark.parametrize("float32", [False, True])
@pytest.mark.parametrize("k_adjacent", [False, True])
def test_few_rows(float32, k_adjacent):
    one = {plans.product(rows, k, cols, None, float32, k_adjacent) for rows, k, cols in plans.FEW}
    grouped = {plans.product(sum(loads) + dropped, k, cols, len(loads), float32, k_adjacent) for loads, dropped, k, cols in plans.FEW_GROUPED}
    assert {"few%d%s" % (r, n) for r in (1, 2, 4) for n in ("", "n", "n/s")} <= grouped
    # (one matrix of floats takes tiles of 64 from 33 rows on; 64 columns and k in parts go together only where columns are adjacent)
    assert {"few%d%s" % (r, n) for r in ((1, 2) if float32 else (1, 2, 4)) for n in ("", "n", "n/s" if k_adjacent else "/s")} <= one

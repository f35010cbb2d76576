"""The sizes that the GPU tests of the dense products run come to every kernel and tile there is, so that no change of the rule that chooses
them leaves one without a test."""
import ctypes
import random

import pytest

import dense_plans as plans
import paper_2007_14152_amd as sp

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


def most(rng, log2):
    return min(int(2 ** rng.uniform(0, log2)) + rng.randint(0, 2), 2 ** log2 - (log2 == 31))


def test_what_is_too_large_is_what_the_header_says():
    """2^24 tiles of 128 x 128 are refused, fewer are not, whatever tiles the sizes come to."""
    rng, size, refused = random.Random(5), ctypes.c_size_t(), 0
    cases = [(1024, 8, n, 1024) for n in ((1 << 21) - 128, (1 << 21) - 127, 1 << 21)] + [(r, 8, 1 << 20, 1024) for r in (900, 2047, 2048, 40000, 131072 * 8)]
    while len(cases) < 4000:
        case = most(rng, 31), most(rng, 30), most(rng, 30), rng.choice([None, 1, 2, 7, 64, 1000, 1024])
        if case[0] * case[2] < 2 ** 45 and case[1] * case[2] * (case[3] or 1) < 2 ** 45:
            cases.append(case)
    for rows, k, cols, experts in cases:
        lines = (rows + 127) // 128 if experts is None else min(rows, rows // 128 + experts + 1)
        tiles = lines * ((cols + 127) // 128)
        for type in (0, 1):
            got = sp.lib().spdnn_linear_bytes(rows, k, cols, experts is not None, experts or 1, type, ctypes.byref(size))
            assert (got != sp.SPDNN_OK) == (tiles >= 2 ** 24), (rows, k, cols, experts, type, tiles)
            refused += got != sp.SPDNN_OK
    assert 50 < refused < 7000

"""The router's reference with its bounds: against the one with plain loops, and as narrow as it has to be where masks put the
type's lowest value, -inf and NaN into a row."""
import numpy as np
import pytest
import torch

import rows_ref as ref

F32, BF16, F16 = ref.TYPES
SCORES = [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)]


def case(rows, experts, k, dtype, score, normalise, masked):
    logits, bias, keep = ref.router_input(rows + experts, rows, experts, dtype, True, masked)
    chosen, is_open = ref.choose_all(logits, k, bias, keep)
    dweight = np.random.default_rng(rows).standard_normal((rows, k)).astype(np.float32).astype(np.float64)
    l = np.where(is_open, ref.f64(logits), -np.inf)
    return logits, bias, keep, l, chosen, is_open, dweight


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("score,normalise", SCORES)
@pytest.mark.parametrize("rows,experts,k", [(5, 3, 2), (40, 30, 16), (31, 256, 8)])
def test_both_references_agree(rows, experts, k, dtype, score, normalise, masked):
    logits, bias, keep, l, chosen, is_open, dw = case(rows, experts, k, dtype, score, normalise, masked)
    first = ref.choose(logits.float().numpy(), k, bias.numpy(), None if keep is None else keep.numpy())
    assert np.array_equal(chosen, first[0]) and np.array_equal(is_open, first[1])
    w, _, d, _ = ref.router(l, is_open, chosen, score, normalise, 2.5, dw)
    assert np.allclose(w, ref.weights(l, is_open, chosen, score, normalise, 2.5), rtol=1e-12, atol=1e-300)
    assert np.allclose(d, ref.route_grad(dw, l, is_open, chosen, score, normalise, 2.5)[0], rtol=1e-10, atol=1e-14)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("score,normalise", SCORES)
def test_bounds_leave_no_room_for_a_wrong_weight(score, normalise, dtype, masked):
    """A weight or an entry of the gradient that is off by one part in a hundred is refused in every row that has one."""
    _, _, _, l, chosen, is_open, dw = case(60, 100, 5, dtype, score, normalise, masked)
    w, bound, d, dbound = ref.router(l, is_open, chosen, score, normalise, 2.5, dw)
    for what, room, out, some in ((w, bound, F32, 0.01), (d, dbound, dtype, 0.02)):
        ref.assert_within(torch.from_numpy(what), what, room, out)
        largest = np.abs(what).argmax(1)
        tried = 0
        for t in range(len(what)):
            if not np.abs(what[t]).max() > 1e-6:
                continue
            off = what.copy()
            off[t, largest[t]] *= 1 + some
            with pytest.raises(AssertionError):
                ref.assert_within(torch.from_numpy(off), what, room, out)
            tried += 1
        assert tried > 30

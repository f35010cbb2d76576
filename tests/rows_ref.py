"""The row operators from their formulas in 64 bits, with plain loops over rows, and how far 32-bit sums may be off.

Every bound is elementwise and follows from the arithmetic alone: U is the unit roundoff of a 32-bit float, a sum of m terms
in any grouping is off by at most m U times the sum of their magnitudes, and an output of fewer bits by its own unit
roundoff on top (half the distance of two neighbours, or half the smallest subnormal).
"""
import numpy as np
import torch

U = 2.0 ** -24
OUT_U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def f64(t):
    return t.detach().cpu().double().numpy()


def assert_within(got, want, bound, dtype, what=""):
    """|got - want| <= bound + rounding of want to dtype; where want is not finite, got is the same."""
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True), what
    off = np.abs(np.where(fin, got - np.where(fin, want, 0), 0))
    room = np.where(fin, bound, 0) * (1 + OUT_U[dtype]) + OUT_U[dtype] * np.abs(np.where(fin, want, 0)) + SMALLEST[dtype]
    bad = ~(off <= room)
    assert not bad.any(), (what, int(bad.sum()), off[bad][:4], room[bad][:4], np.argwhere(bad)[:4])


def embed_grad(dout, ids, vocab, scale, base=None):
    """(gradient, bound): dout float64 [n, width], ids int64 [n]."""
    total = np.zeros((vocab, dout.shape[1]))
    size = np.zeros_like(total)
    many = np.zeros((vocab, 1))
    for t, i in enumerate(ids):
        if 0 <= i < vocab:
            total[i] += dout[t]
            size[i] += np.abs(dout[t])
            many[i] += 1
    bound = (many + 2) * U * size * abs(scale)
    total = total * scale
    if base is not None:
        bound = bound + 2 * U * np.abs(base)
        total = total + base
    return total, bound


def choose(logits32, k, bias32=None, keep=None):
    """chosen int32 [rows, k], open bool [rows, experts]; the sum is one of 32-bit floats by definition."""
    rows, experts = logits32.shape
    with np.errstate(all="ignore"):
        r = logits32 if bias32 is None else (logits32 + bias32).astype(np.float32)
        is_open = r > -np.inf
    if keep is not None:
        is_open &= keep[:, None]
    chosen = np.full((rows, k), -1, dtype=np.int32)
    for t in range(rows):
        order = sorted((e for e in range(experts) if is_open[t, e]), key=lambda e: (-r[t, e], e))[:k]
        chosen[t, :len(order)] = order
    return chosen, is_open


def sigmoid(x):
    with np.errstate(all="ignore"):
        return np.where(x >= 0, 1 / (1 + np.exp(-x)), np.exp(x) / (1 + np.exp(x)))


def log_sigmoid(x):
    with np.errstate(all="ignore"):
        return np.minimum(x, 0) - np.log1p(np.exp(-np.abs(x)))


def weights(logits, is_open, chosen, score, normalise, scale):
    """Weights in 64 bits; logits float64."""
    rows, k = chosen.shape
    w = np.zeros((rows, k))
    with np.errstate(all="ignore"):
        for t in range(rows):
            at = chosen[t][chosen[t] >= 0]
            if len(at) == 0:
                continue
            l = logits[t, at]
            if normalise:
                x = l if score == "softmax" else log_sigmoid(l)
                e = np.exp(x - x.max())
                w[t, :len(at)] = e / e.sum()
            elif score == "softmax":
                x = logits[t, is_open[t]]
                w[t, :len(at)] = np.exp(l - x.max()) / np.exp(x - x.max()).sum()
            else:
                w[t, :len(at)] = sigmoid(l)
    return w * scale


def weight_slack(logits, is_open, experts):
    """Relative error of a weight, per row: of its exponent, which is rounded at the size of the logits (twice: the shift, and
    log_sigmoid before it), of a few functions of 2 ulp each, and of a sum of at most `experts` positive terms."""
    size = np.where(is_open & np.isfinite(logits), np.abs(logits), 0).max(1, keepdims=True, initial=0)
    return (4 * size + experts + 24) * U


def route_grad(dweight, logits, is_open, chosen, score, normalise, scale):
    """(gradient, bound)."""
    rows, experts = logits.shape
    d = np.zeros((rows, experts))
    bound = np.zeros((rows, experts))
    rel = weight_slack(logits, is_open, experts)
    one = weights(logits, is_open, chosen, score, normalise, 1.0)
    for t in range(rows):
        valid = chosen[t] >= 0
        at = chosen[t][valid]
        if len(at) == 0:
            continue
        g = dweight[t, valid] * scale
        w = one[t, valid]
        mean, size = (g * w).sum(), (np.abs(g) * w).sum()
        if score == "softmax" and not normalise:
            o = np.nonzero(is_open[t])[0]
            x = logits[t, o]
            p = np.exp(x - x.max())
            p /= p.sum()
            spread = np.zeros(experts)
            spread[at] = g
            d[t, o] = p * (spread[o] - mean)
            bound[t, o] = 3 * rel[t] * p * (np.abs(spread[o]) + size)
            continue
        if normalise:
            v, b = w * (g - mean), w * (np.abs(g) + size)
            if score == "sigmoid":
                v, b = v * sigmoid(-logits[t, at]), b * sigmoid(-logits[t, at])
        else:
            v = g * w * sigmoid(-logits[t, at])
            b = np.abs(v)
        d[t, at] = v
        bound[t, at] = 3 * rel[t] * b
    return d, bound


def sort_pairs(chosen, experts):
    """(place int32 [rows, k], offsets int32 [experts + 1])."""
    flat = chosen.reshape(-1)
    lists = [[] for _ in range(experts)]
    for p, e in enumerate(flat):
        if 0 <= e < experts:
            lists[e].append(p)
    place = np.full(flat.shape, -1, dtype=np.int32)
    offsets = np.zeros(experts + 1, dtype=np.int32)
    at = 0
    for e in range(experts):
        for p in lists[e]:
            place[p] = at
            at += 1
        offsets[e + 1] = at
    return place.reshape(chosen.shape), offsets


def combine(ys, place, weight, add):
    """(out, bound)."""
    rows, k = place.shape
    out = np.zeros((rows, ys.shape[1]))
    size = np.zeros_like(out)
    for t in range(rows):
        for j in range(k):
            if 0 <= place[t, j] < rows * k:
                y = ys[place[t, j]] * (1.0 if weight is None else weight[t, j])
                out[t] += y
                size[t] += np.abs(y)
    if add is not None:
        out += add
        size += np.abs(add)
    return out, (k + 2) * U * size


# ---------------------------------------------------------------------------
# the router, all rows at once, with bounds that logits far below a row's largest do not widen
# ---------------------------------------------------------------------------
FAR = 110.0  # exp(-FAR) is less than half the smallest float
TINY = SMALLEST[torch.float32]


def router_input(seed, rows, experts, dtype, with_bias, masked):
    """(logits, bias, keep) on the CPU.  masked: three tenths of the logits are -inf, or NaN in every fifth row, every seventh
    column holds the type's lowest value (open, but last), and a fifth of the rows go to no expert."""
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(rows, experts, generator=g) * 2).to(dtype)
    bias = torch.randn(experts, generator=g) if with_bias else None
    if not masked:
        return logits, bias, None
    off = torch.rand(rows, experts, generator=g) < 0.3
    logits[off] = -float("inf")
    logits[:, ::7] = torch.finfo(dtype).min
    logits[::5] = torch.where(off[::5], float("nan"), logits[::5])
    return logits, bias, torch.rand(rows, generator=g) < 0.8


def choose_all(logits, k, bias=None, keep=None):
    """choose for tensors of many rows: (chosen int32 [rows, k], open bool [rows, experts]) as arrays."""
    r = logits.float().cpu()
    if bias is not None:
        r = r + bias.cpu()
    is_open = r > -float("inf")
    if keep is not None:
        is_open &= keep.cpu()[:, None]
    at = torch.sort(torch.where(is_open, r, -float("inf")), dim=1, descending=True, stable=True).indices[:, :k]
    return torch.where(is_open.gather(1, at), at, -1).int().numpy(), is_open.numpy()


def router(logits, is_open, chosen, score, normalise, scale, dweight):
    """(weights, bound, gradient, bound); logits and dweight float64.

    A weight is off by its exponent, which is rounded at the size of the difference D to the largest logit (and by log_sigmoid,
    at the size Y of its value, on either side of that difference), by exp and log1p (4 U each), by the sum of m positive terms
    (m U, and by what its terms are off), by the quotient and the scale.  Only terms within FAR of the largest count: the others
    are zeros, or a few of the smallest floats.  A logit beyond 200 is its own log_sigmoid, exactly.  The gradient is a product
    of a weight and a difference of terms that hold another, k of them added."""
    rows, experts = logits.shape
    k = chosen.shape[1]
    valid = chosen >= 0
    at = np.where(valid, chosen, 0)
    with np.errstate(all="ignore"):
        L = np.where(is_open, logits, -np.inf)
        picked = np.where(valid, np.take_along_axis(L, at, 1), -np.inf)
        everything = score == "softmax" and not normalise
        if score == "sigmoid" and not normalise:
            w = np.where(valid, sigmoid(picked), 0.0)
            rel = np.full((rows, 1), 16.0)
        else:
            x, there = (L, is_open) if everything else (picked if score == "softmax" else log_sigmoid(picked), valid)
            top = np.where(there, x, -np.inf).max(1, keepdims=True)
            below = np.where(there, x - np.where(np.isfinite(top), top, 0.0), -np.inf)
            e = np.exp(below)
            total = e.sum(1, keepdims=True)
            p = e / np.where(total > 0, total, 1.0)
            near = there & (below > -FAR)
            rel = 2 * np.where(near, -below, 0.0).max(1, keepdims=True) + x.shape[1] + 16
            if score == "sigmoid":
                rel = rel + 32 + 4 * np.where(near & (np.abs(picked) < 200), np.abs(x), 0.0).max(1, keepdims=True)
            w = np.where(valid, np.take_along_axis(p, at, 1), 0.0) if everything else p
        bound = 1.001 * rel * U * w * scale + 4 * TINY * max(1.0, scale)
        g = np.where(valid, np.where(valid, dweight, 0.0) * scale, 0.0)
        mean, size, most = (g * w).sum(1, keepdims=True), (np.abs(g) * w).sum(1, keepdims=True), np.abs(g).sum(1, keepdims=True)
        d = np.zeros((rows, experts + 1))
        dbound = np.zeros_like(d)
        slot = np.where(valid, chosen, experts)
        if everything:
            spread = np.zeros_like(d)
            np.put_along_axis(spread, slot, g, 1)
            spread = spread[:, :-1]
            any_slot = valid.any(1, keepdims=True)
            d = np.where(any_slot, p * (spread - mean), 0.0)
            dbound = np.where(any_slot, 1.001 * (2 * rel + k + 40) * U * p * (np.abs(spread) + size) + 8 * TINY * (np.abs(spread) + most + 1), 0.0)
            return w * scale, bound, d, dbound
        if normalise:
            v, b = w * (g - mean), (2 * rel + k + 40) * U * w * (np.abs(g) + size)
            if score == "sigmoid":
                v, b = v * sigmoid(-picked), b * sigmoid(-picked)
        else:
            v = g * w * sigmoid(-picked)
            b = 40 * U * np.abs(v)
        v, b = np.where(valid, v, 0.0), np.where(valid, 1.001 * b + 8 * TINY * (np.abs(g) + most + 1), 0.0)
        np.put_along_axis(d, slot, v, 1)
        np.put_along_axis(dbound, slot, b, 1)
        return w * scale, bound, d[:, :-1], dbound[:, :-1]

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

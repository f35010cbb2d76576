"""The dense products and layer norm from their formulas in 64 bits, and how far 32-bit sums may be off.

U is the unit roundoff of a 32-bit float.  A matrix instruction may cut off where an addition rounds, so a sum of m terms in any
grouping is off by at most 2 m U times the sum of their magnitudes; an output of fewer bits is off by its own unit roundoff on top
(rows_ref.assert_within adds that).
"""
import math

import torch

from rows_ref import OUT_U, SMALLEST, TYPES, U, assert_within  # noqa: F401  (what the tests of these operators use too)

ACTS = [None, "relu", "clip", "gelu", "silu"]


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "clip":
        return z.clamp(0, 32)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "clip":
        return ((z > 0) & (z < 32)).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


# How far the activations and slopes that are computed in 32 bits are off for an argument z.  gelu: the product with 1 / sqrt 2 is
# off by 2 U, which moves erf by 2 U max(t erf'(t)) < U; erf itself is off by 4 U, the sum and the products by 3 U, all of it times
# |z|.  The slope has z exp(-z^2 / 2) besides, at most 0.61: its argument is off by 2 U z^2 / 2, z^3 exp(-z^2 / 2) is at most 1.16,
# and exp and three products by 7 U.  silu: exp is off by 4 U, sum and quotient by 2 U.
def act_off(z, name):
    return 8 * U * z.abs() if name in ("gelu", "silu") else torch.zeros_like(z)


def slope_off(z, name):
    if name == "gelu":
        return torch.full_like(z, 16 * U)
    if name == "silu":
        return 16 * U * (1 + z.abs() * torch.sigmoid(z) * torch.sigmoid(-z))
    return torch.zeros_like(z)


STEEPEST = {None: 1.0, "relu": 1.0, "clip": 1.0, "gelu": 1.13, "silu": 1.1}


def batches(rows, offsets):
    if offsets is None:
        return [(0, 0, rows)]
    at = offsets.tolist()
    return [(e, at[e], at[e + 1]) for e in range(len(at) - 1)]


def linear(x, weight, bias=None, name=None, add=None, offsets=None):
    """(out, bound, pre, its bound) of tensors on the CPU, in 64 bits."""
    rows, width = x.shape
    cols = weight.shape[-1]
    z, zoff, out, off = (torch.zeros(rows, cols, dtype=torch.float64) for _ in range(4))
    for e, a, b in batches(rows, offsets):
        w = (weight if offsets is None else weight[e]).double()
        r = slice(a, b)
        z[r] = x[r].double() @ w
        zoff[r] = 2 * (width + 1) * U * (x[r].double().abs() @ w.abs())
        if bias is not None:
            v = (bias if offsets is None else bias[e]).double()
            z[r] += v
            zoff[r] += 2 * U * (z[r].abs() + v.abs())
        out[r] = act(z[r], name)
        off[r] = STEEPEST[name] * zoff[r] + act_off(z[r], name)
        if add is not None:
            out[r] += add[r].double()
            off[r] += U * (out[r].abs() + off[r])
    return out, off, z, zoff


def linear_grad(dout, x, weight, pre=None, name=None, offsets=None):
    """(dx, dweight, dbias) and their bounds; d is rounded to x's type where there is an activation or dout has another type."""
    rows, width = x.shape
    cols = weight.shape[-1]
    d = dout.double()
    doff = torch.zeros_like(d)
    if name is not None:
        s = slope(pre.double(), name)
        doff = d.abs() * slope_off(pre.double(), name) + U * (d * s).abs()
        d = d * s
    if name is not None or dout.dtype != x.dtype:
        doff = doff * (1 + OUT_U[x.dtype]) + OUT_U[x.dtype] * d.abs() + SMALLEST[x.dtype]
    dx, dxoff = torch.zeros(rows, width, dtype=torch.float64), torch.zeros(rows, width, dtype=torch.float64)
    sets = () if offsets is None else (weight.shape[0],)
    dw, dwoff = torch.zeros(sets + (width, cols), dtype=torch.float64), torch.zeros(sets + (width, cols), dtype=torch.float64)
    db, dboff = torch.zeros(sets + (cols,), dtype=torch.float64), torch.zeros(sets + (cols,), dtype=torch.float64)
    for e, a, b in batches(rows, offsets):
        if a == b:
            continue
        at = (Ellipsis,) if offsets is None else (e,)
        w, xr, dr, dof = weight[at].double(), x[a:b].double(), d[a:b], doff[a:b]
        dx[a:b] = dr @ w.t()
        dxoff[a:b] = (dof + 2 * (cols + 1) * U * (dr.abs() + dof)) @ w.abs().t()
        dw[at] = xr.t() @ dr
        dwoff[at] = xr.abs().t() @ (dof + 2 * (b - a + 1) * U * (dr.abs() + dof))
        db[at] = dr.sum(0)
        dboff[at] = (dof + 2 * (b - a + 1) * U * (dr.abs() + dof)).sum(0)
    return (dx, dw, db), (dxoff, dwoff, dboff)


def norm(x, weight=None, bias=None, eps=1e-5):
    """(out, bound, mean, rstd, bounds of both).  The mean of w numbers is off by (w + 2) U times their mean magnitude m.  A
    difference from it is off by that and U of itself; the variance v, a mean of squares, by twice the differences' error times their
    mean magnitude (at most sqrt v), that error's square, and (w + 4) U of itself; rstd by half the relative error of v + eps, and 4 U."""
    x = x.double()
    w = x.shape[1]
    mean = x.mean(1, keepdim=True)
    mean_off = (w + 2) * U * x.abs().mean(1, keepdim=True)
    d = x - mean
    v = (d * d).mean(1, keepdim=True)
    e = mean_off + U * v.sqrt()
    v_off = 2 * e * v.sqrt() + e * e + (w + 4) * U * v
    rstd = 1 / torch.sqrt(v + eps)
    rel = 0.5 * v_off / (v + eps) * (1 + v_off / (v + eps)) ** 2 + 4 * U
    rstd_off = rstd * rel
    h = d * rstd
    h_off = (mean_off + U * d.abs()) * rstd * (1 + rel) + h.abs() * (rel + U)
    out, off = h, h_off
    if weight is not None:
        off = (off + U * (h.abs() + off)) * weight.double().abs()
        out = out * weight.double()
    if bias is not None:
        out = out + bias.double()
        off = off + U * (out.abs() + off)
    return out, off, mean, rstd, mean_off, rstd_off


def norm_grad(dout, x, stats, weight=None, add=None):
    """(dx, dweight, dbias) and bounds, of the stats that are given (two floats a row)."""
    mean, rstd = stats[:, :1].double(), stats[:, 1:].double()
    dout = dout.double()
    n, w = x.shape
    h = (x.double() - mean) * rstd
    h_off = 2 * U * h.abs()
    g = dout if weight is None else dout * weight.double()
    gh = g * h
    gh_off = 5 * U * gh.abs()
    a, b = g.mean(1, keepdim=True), gh.mean(1, keepdim=True)
    a_off = (w + 3) * U * g.abs().mean(1, keepdim=True)
    b_off = (w + 6) * U * gh.abs().mean(1, keepdim=True)
    dx = rstd * (g - a - h * b)
    off = rstd * (U * g.abs() + a_off + h.abs() * b_off + 4 * U * (h * b).abs()) + 4 * U * rstd * (g.abs() + a.abs() + (h * b).abs())
    if add is not None:
        dx = dx + add.double()
        off = off + U * (dx.abs() + off)
    dh = dout * h
    dw, dw_off = dh.sum(0), (n + 6) * U * dh.abs().sum(0)
    db, db_off = dout.sum(0), (n + 2) * U * dout.abs().sum(0)
    return (dx, dw, db), (off, dw_off, db_off)

"""Plain 64-bit forms of the dense operators and how far an implementation with fp32 sums may be from them.

Tolerances.  u = 2^-24.  A sum of K products in fp32, in any order, is off by at most (K + 1) u sum |terms|; matrix
instructions that truncate where they add count twice, so 2 (K + 2) u sum |terms| is allowed before the activation.  An
activation passes on at most 1.13 times that (the steepest is gelu's) and adds errors of its own, 16 u of the value and of |z|
(exp and erfc are good to a few units).  The result is rounded to its type by half a step, eps / 2 of its value, plus half of
the smallest number below the normal range.
"""
import math

import torch

U = 2.0 ** -24
ACTS = ("none", "relu", "gelu", "silu", "sigmoid")


def act64(z, act):
    if act == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return 1 / (1 + torch.exp(-z)) if act == "sigmoid" else z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    if act == "silu":
        return s + z * s * (1 - s)
    return s * (1 - s) if act == "sigmoid" else torch.ones_like(z)


def rounding(x, dtype):
    return torch.finfo(dtype).eps / 2 * x.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def ranges(offsets, groups, rows):
    """Rows of each group: running maximum of the clamped offsets."""
    if offsets is None:
        return [(0, rows)]
    top, out = 0, []
    o = [min(max(int(v), 0), rows) for v in offsets.tolist()]
    for g in range(groups):
        top = max(top, o[g])
        out.append((top, max(top, o[g + 1])))
    return out


def forward64(x, w, bias=None, residual=None, act="none", offsets=None):
    """(out, tolerance, z, tolerance of z) with NaN in rows of no group."""
    rows, (n, k) = x.shape[0], w.shape[-2:]
    dtype = x.dtype
    ws, x = (w if offsets is not None else w[None]).double(), x.double()
    bs = None if bias is None else (bias if offsets is not None else bias[None]).double()
    z = torch.full((rows, n), math.nan, dtype=torch.float64)
    size = z.clone()
    for g, (lo, hi) in enumerate(ranges(offsets, ws.shape[0], rows)):
        z[lo:hi] = x[lo:hi] @ ws[g].t() + (0 if bs is None else bs[g])
        size[lo:hi] = x[lo:hi].abs() @ ws[g].abs().t() + (0 if bs is None else bs[g].abs())
    tz = 2 * (k + 2) * U * size
    y = act64(z, act)
    r = residual.double() if residual is not None else torch.zeros_like(z)
    out = y + r
    tol = 1.13 * tz + 16 * U * (y.abs() + z.abs() + r.abs() + (act == "sigmoid")) + rounding(out, dtype)
    return out, tol, z, tz + rounding(z, dtype)


def backward64(x, w, grad, pre=None, act="none", offsets=None):
    """(dx, dw, dbias) and their tolerances, from the stored pre-activation; NaN in dx's rows of no group.  dz is rounded to
    the type before the products, half a step of each term."""
    dtype, rows, (n, k) = x.dtype, x.shape[0], w.shape[-2:]
    ws, x, grad = (w if offsets is not None else w[None]).double(), x.double(), grad.double()
    dz = grad if act == "none" else grad * slope64(pre.double(), act)
    ez = torch.zeros_like(dz) if act == "none" else rounding(dz, dtype) + 32 * U * grad.abs() * (1 + pre.double().abs())
    dx, tx = torch.full((rows, k), math.nan, dtype=torch.float64), torch.zeros(rows, k, dtype=torch.float64)
    dw, db = torch.zeros_like(ws), torch.zeros(ws.shape[:2], dtype=torch.float64)
    tw, tb = torch.zeros_like(dw), torch.zeros_like(db)
    for g, (lo, hi) in enumerate(ranges(offsets, ws.shape[0], rows)):
        d, e, m = dz[lo:hi], ez[lo:hi], hi - lo
        size = d.abs() + e
        dx[lo:hi], tx[lo:hi] = d @ ws[g], e @ ws[g].abs() + 2 * (n + 2) * U * (size @ ws[g].abs())
        dw[g], tw[g] = d.t() @ x[lo:hi], e.t() @ x[lo:hi].abs() + 2 * (m + 2) * U * (size.t() @ x[lo:hi].abs())
        db[g], tb[g] = d.sum(0), e.sum(0) + 2 * (m + 2) * U * size.sum(0)
    tx, tw, tb = tx + rounding(dx, dtype), tw + rounding(dw, dtype), tb + rounding(db, dtype)
    if offsets is None:
        dw, db, tw, tb = dw[0], db[0], tw[0], tb[0]
    return (dx, dw, db), (tx, tw, tb)


def ortho(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, dtype=torch.float64):
    """Newton-Schulz steps on [batch, rows, cols], in 64 bits or in another type (the norm always in 64)."""
    c = [tuple(coefficients)] * steps if not isinstance(coefficients[0], (tuple, list)) else coefficients
    x = g.double()
    x = (x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)).to(dtype)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for a, b, q in c:
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + q * (A @ A)) @ x
    return x.transpose(1, 2) if tall else x


def check_ortho(got, g, what, **how):
    """Relative 2-norm, matrix by matrix: at most three times what the same formula in fp32 is off, and the rounding to the type.
    (Errors grow up to 485 times in five steps where singular values are small, in any implementation with fp32 sums: it is
    the formula in 32 bits, on these inputs, that says how much.)"""
    want, single = ortho(g, **how), ortho(g, dtype=torch.float32, **how).double()
    got = got.double()
    for z in range(g.shape[0]):
        norm = want[z].norm()
        off, ref = (got[z] - want[z]).norm(), (single[z] - want[z]).norm()
        most = 3 * ref + (torch.finfo(g.dtype).eps / 2 + 8 * U) * norm + 1e-30
        assert off <= most, "%s, matrix %d: off by %.3g of %.3g, allowed %.3g" % (what, z, off, norm, most)


def check(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError("%s: %d of %d outside, first at %s: %r, want %r +- %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(tol[i])))

"""Plain 64-bit forms of layer norm, embedding lookup and the stable embedding with
their gradients, and how far a computation in fp32 that rounds its results once may be
from them.

The bounds count roundings.  U = 2^-24 is half a step of fp32, HALF[t] half a step of
the type a result is stored in.  A sum of n terms in fp32, whatever its tree, is off
by at most depth * U * sum |terms|, where depth is the largest number of additions
that one term goes through.  `depth` allows for what the kernels do and more: parts of a
few hundred terms one after the other, then trees.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def depth(n):
    return min(n, 160 + n / 256)


def layer_norm(x, w, b, eps):
    """(y, xh, mean, rstd) in 64 bits; x a matrix of rows, w and b may be None."""
    x = x.double()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / (xc.square().mean(1, keepdim=True) + eps).sqrt()
    xh = xc * rstd
    y = xh if w is None else xh * w.double()
    return (y if b is None else y + b.double()), xh, mean, rstd


def xh_error(xh, n):
    """Of xh in fp32: the mean is corrected by the mean of x - mean, so its error counts
    against that (|xh| averages at most 1); rstd's error is half of the variance's."""
    d = depth(n)
    return U * (d + (d / 2 + 8) * xh.abs())


def forward_bound(y, xh, w, dtype, n):
    e = xh_error(xh, n)
    if w is not None:
        e = e * w.double().abs() + U * (xh * w.double()).abs()
    return e + (2 * U + HALF[dtype]) * y.abs() + TINY[dtype]


def layer_norm_grads(dy, xh, rstd, w):
    """(dx, dw, db) in 64 bits."""
    dy = dy.double()
    g = dy if w is None else dy * w.double()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def backward_bounds(dy, xh, mean, rstd, w, dx, dw, db, dtype, pdtype, dy_error=0.0):
    """Bounds of (dx, dw, db); dy_error: how far dy itself may be off, elementwise."""
    m, n = dy.shape
    d = depth(n)
    dy = dy.double().abs()
    wa = torch.ones((), dtype=torch.float64, device=dy.device) if w is None else w.double().abs()
    # a saved mean is rounded once
    xe = xh_error(xh, n) + U * mean.abs() * rstd
    g, ge = dy * wa, (dy_error + U * dy) * wa
    c1, c2 = g.mean(1, keepdim=True), (g * xh.abs()).mean(1, keepdim=True)
    c1e = d * U * c1 + ge.mean(1, keepdim=True)
    c2e = (d + 2) * U * c2 + (g * xe + ge * xh.abs()).mean(1, keepdim=True)
    inner = g + c1 + xh.abs() * c2
    e = rstd * (ge + c1e + xh.abs() * c2e + xe * c2 + 4 * U * inner)
    dxe = e + (d / 2 + 8) * U * rstd * inner + HALF[dtype] * dx.abs() + TINY[dtype]
    r = depth(m) + 4
    dwe = (r * U * (dy * xh.abs()) + dy * xe + dy_error * xh.abs()).sum(0)
    dbe = (r * U * dy + dy_error).sum(0)
    return (dxe, dwe + HALF[pdtype] * dw.abs() + TINY[pdtype],
            dbe + HALF[pdtype] * db.abs() + TINY[pdtype])


def row_sums(dy, ids, num):
    """Sums of dy's rows by id, of their magnitudes, and the counts, in 64 bits; ids outside
    of [0, num) are left out."""
    ids = ids.reshape(-1).long()
    dy = dy.reshape(ids.numel(), -1).double()
    keep = (ids >= 0) & (ids < num)
    ids, dy = ids[keep], dy[keep]
    s = torch.zeros(num, dy.shape[1], dtype=torch.float64, device=dy.device)
    a = torch.zeros_like(s)
    s.index_add_(0, ids, dy)
    a.index_add_(0, ids, dy.abs())
    return s, a, torch.bincount(ids, minlength=num)


def sum_error(a, count):
    """Of a row's sum in fp32: a its sum of magnitudes, count its terms, added in parts of 64
    one after the other, then the parts."""
    c = count.double()[:, None]
    return U * a * torch.minimum(c, 256 + c / 64)


def check(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, what
    over = ((got - want).abs() - bound)
    bad = ~(over <= 0)
    if bool(bad.any()):
        i = int(torch.argmax(torch.where(bad, over, torch.full_like(over, -1.0)).nan_to_num(
            1e300).reshape(-1)))
        raise AssertionError(
            f"{what}: {int(bad.sum())} of {bad.numel()} values outside; at {i}: "
            f"{float(got.reshape(-1)[i])!r} for {float(want.reshape(-1)[i])!r}, bound "
            f"{float(bound.expand_as(want).reshape(-1)[i]):.3g}")

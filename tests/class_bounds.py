"""How far the class losses may be from their definition, pair by pair of a row and a class: a bound that shrinks with p - q.

Beside class_util.bounds, which allows a gradient an error of a share of p + q (and so any gradient at all to a row that has
learned its class), and which lets the largest row and the largest class of the tables count for all.  With u as there:
  a score z[t,v]    (D + 4) 2^-24 A[t,v] for A = s sum |h||w|, nothing where `exact` says that every product and sum is a
                    number of its type; fp32 tables 3 * 2^-22 A more, and 2^-38 D of the largest elements of this row and this
                    class.  To the base 2 and with the running reference taken off: 8 * 2^-24 |z|
  the log-sum-exp   its scores' errors, each with its share p of the sum; (V / 16 + 64) 2^-24 for the sum, 8 * 2^-24 |lse|
  p[t,v]            (error of z and of the log-sum-exp + 2^-20) of itself
  a gradient        u |p - q| where P, less what a slot takes, is rounded to 16 bits (p - q is formed in fp32 and then rounded
                    wherever a slot names the class, p alone elsewhere); the error of p; fp32 sums of n terms, (n + 80) 2^-24
                    (p + q); fp16 planes end at 2^-24 of what is at most 2^15, where at least 2^14 stands for the largest
                    term: 2^-38 of that a term
"""
from __future__ import annotations

import torch

from class_util import U_P

TINY = 2.0 ** -24


def _sum(p, e):
    """Sum over classes of p * e, in which a class without any share counts nothing, infinite as its error may be."""
    return torch.where(p > 0, p * e, 0.0)


def bounds(dtype, x, g=None, exact=False):
    """The bounds of class_util.reference()'s results, from what it returns beside them."""
    h, w, s, p, q, lse = x["h"].abs(), x["w"].abs(), x["s"], x["p"], x["q"], x["lse"].abs()[:, None]
    (T, D), V = h.shape, w.shape[0]
    a = h @ w.T * s
    dz = torch.zeros_like(a) if exact else (D + 4) * TINY * a
    if dtype == "f32" and not exact:
        dz = dz + 3 * 2.0 ** -22 * a + 2.0 ** -38 * D * s * h.amax(1, keepdim=True) * w.amax(1)
    dz = dz + 8 * TINY * x["z"].abs()
    dlse = _sum(p, dz).sum(1, keepdim=True) + (V / 16 + 64) * TINY + 8 * TINY * lse
    own = _sum(q, dz).sum(1, keepdim=True)
    b = {"lse": dlse[:, 0], "loss": (dlse + own + 16 * TINY * (lse + _sum(q, x["z"].abs()).sum(1, keepdim=True) + 64))[:, 0]}
    share = U_P[dtype] * (p - q).abs() + _sum(p, dz + dlse + 2.0 ** -20)
    row = share + (V + 80) * TINY * (p + q)
    b["row_grad"] = s * (row @ w)
    if dtype == "f16":
        b["row_grad"] = b["row_grad"] + s * 2.0 ** -38 * w.sum(0)
    elif dtype == "f32":
        b["row_grad"] = b["row_grad"] + s * 2.0 ** -38 * (p > 0).sum(1, keepdim=True) * _sum(p, w.amax(1)).amax(1, keepdim=True)
    if g is not None:
        g = torch.where(x["some"], g.double().abs(), 0.0)[:, None]
        b["grad_h"] = g * (b["row_grad"] + s * TINY * (row @ w))
        b["grad_w"] = s * ((g * (share + (T + 80) * TINY * (p + q))).T @ h)
        if dtype == "f16":
            b["grad_w"] = b["grad_w"] + s * 2.0 ** -38 * g.amax() * h.sum(0)
        elif dtype == "f32":
            b["grad_w"] = b["grad_w"] + s * 2.0 ** -38 * T * (g * h.amax(1, keepdim=True)).amax()
    return b

"""The block's operators in 64 bits, each result with a bound of its error that follows from the roundings on the way.

u is half a step of the type (bfloat16 2^-8, fp16 2^-11, fp32 2^-24), v that of fp32.  A sum of n products in fp32 is off by at most
n v times the sum of their magnitudes; fp32 operands of a product are taken as three planes of 8 bits, of whose nine products
the three smallest (3 * 2^-24 of each product) are left out.  fp16 has no finer step than 2^-24, so that nothing is rounded
better than 2^-25.
"""
import math

import torch

V = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FLOOR = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def rounding(x, dtype):
    """What rounding to the type adds to an error: half a step of the value."""
    return HALF_STEP[dtype] * x.abs() + FLOOR[dtype]


def product(a, b, ea=0.0, eb=0.0, dtype=torch.float32):
    """a b^T with its bound, for operands off by ea and eb."""
    n = a.shape[1]
    size = a.abs() @ b.abs().mT.contiguous()
    bound = (n + 8) * V * size
    if isinstance(ea, torch.Tensor):
        bound = bound + ea @ (b.abs() + eb).mT.contiguous()
    if isinstance(eb, torch.Tensor):
        bound = bound + a.abs() @ eb.mT.contiguous()
    return a @ b.mT.contiguous(), bound


def activation(name, g):
    """act, act', and the largest |act'| and |act''|."""
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)), 1.1, 0.5
    if name == "gelu":
        p = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        bell = torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        return g * p, p + g * bell, 1.13, 0.8
    return g.clamp_min(0), (g > 0).double(), 1.0, 0.0


def gated(x, wg, wu, wd, gy, act, dtype):
    """{name: (value, bound)} of the block and its gradients."""
    x, wg, wu, wd = (t.detach().double() for t in (x, wg, wu, wd))
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    if dtype != torch.float32:                               # what a forward keeps for its backward has 24 bits, 16 of them the number's
        eg, eu = eg + 2.0 ** -17 * g.abs(), eu + 2.0 ** -17 * u.abs()
    a, slope, steep, bend = activation(act, g)
    # the functions themselves: exponential and reciprocal within 4 v of their value and (1 + |g|) v of the argument's
    # rounding; the error function within 4 v of one
    ea = steep * eg + (8 + g.abs()) * V * (g.abs() if act != "relu" else 0)
    es = bend * eg + ((8 + g.abs() ** 2) * 2 * V if act != "relu" else (g.abs() <= eg).double())
    h = a * u
    exact_h = ea * (u.abs() + eu) + a.abs() * eu + V * h.abs()
    eh = exact_h + (0 if dtype == torch.float32 else rounding(h, dtype))
    y, ey = product(h, wd, eh)
    out = {"y": (y, ey + rounding(y, dtype))}
    if gy is None:
        return out
    gy = gy.detach().double()
    dh, edh = product(gy, wd.mT.contiguous())
    dg, du = dh * u * slope, dh * a
    edg = edh * (u.abs() + eu) * (slope.abs() + es) + dh.abs() * (eu * (slope.abs() + es) + u.abs() * es) + 3 * V * dg.abs()
    edu = edh * (a.abs() + ea) + dh.abs() * ea + 2 * V * du.abs()
    if dtype == torch.bfloat16:
        edg, edu = edg + rounding(dg, dtype), edu + rounding(du, dtype)
    if dtype == torch.float16:                               # kept beside a power of two of the largest gradient
        top = gy.abs().max().item()
        lift = 2.0 ** -math.floor(math.log2(top)) if top > 0 else 1.0
        edg, edu = edg + rounding(dg * lift, dtype) / lift, edu + rounding(du * lift, dtype) / lift
    t = lambda m: m.mT.contiguous() if isinstance(m, torch.Tensor) else m
    p, ep = product(dg, t(wg), edg)
    q, eq = product(du, t(wu), edu)
    out["grad_x"] = (p + q, ep + eq + rounding(p + q, dtype))
    for name, d, e in (("grad_gate", dg, edg), ("grad_up", du, edu)):
        p, ep = product(t(d), t(x), t(e))
        out[name] = (p, ep + rounding(p, dtype))
    p, ep = product(t(gy), t(h), 0.0, t(eh))
    out["grad_down"] = (p, ep + rounding(p, dtype))
    return out


def norm(x, r, w, gy, gs, eps, dtype):
    """{name: (value, bound)} of the norm and its gradients.  A lane sums 16 elements, shuffles and waves join in 10 more."""
    s = x.detach().double() if r is None else (x.detach().float() + r.detach().float()).to(dtype).double()
    t, d = s.shape
    wd = w.detach().double()
    rstd = (s.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    unit = s * rstd
    out = {"s": (s, torch.zeros_like(s)), "y": (unit * wd, 20 * V * (unit * wd).abs() + rounding(unit * wd, dtype))}
    if gy is None and gs is None:
        return out
    gy = torch.zeros_like(s) if gy is None else gy.detach().double()
    gs = torch.zeros_like(s) if gs is None else gs.detach().double()
    inner, size = (gy * wd * unit).mean(1, keepdim=True), (gy * wd * unit).abs().mean(1, keepdim=True)
    gx = gs + rstd * (gy * wd - unit * inner)
    out["grad_x"] = (gx, 60 * V * (gs.abs() + rstd * ((gy * wd).abs() + unit.abs() * size)) + rounding(gx, dtype))
    gw = (gy * unit).sum(0)
    out["grad_weight"] = (gw, (20 + t) * V * (gy * unit).abs().sum(0) + rounding(gw, w.dtype))
    return out


def check(name, got, value, bound):
    """Every element within its bound; NaN and infinities have none.  A value that its type cannot hold (65520 and more in fp16:
    the largest number and half a step) rounds to an infinity of its sign."""
    assert got.shape == value.shape, name
    got = got.detach()
    beyond = value.abs() + bound > torch.finfo(got.dtype).max
    right = got.double() == value.sign() * math.inf
    off = torch.where(beyond & right, 0.0, (got.double() - value).abs() - bound)
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0.0, "%s: %.3g beyond its bound, at %s" % (name, worst, tuple(int(i) for i in (off == off.max()).nonzero()[0]))
    assert (torch.isfinite(got) | beyond).all(), name

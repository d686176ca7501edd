"""The class losses by their definition in 64 bits, and how far the kernels' results may be from it.

Bounds, with u the unit roundoff of the 16-bit type that probabilities are rounded to (2^-8 bfloat16, 2^-11 fp16, 2^-22 for
the two fp16 planes of fp32 tables):
  a score        fp32 sums of D products: (D + 4) 2^-24 A, A = scale * sum |h||w|; fp32 tables lose 3 * 2^-22 A more (two
                 elements of 22 bits and the lo*lo product) and 2^-38 of (largest |h|)(largest |w|) D for elements far below
                 their table's largest
  a loss         the errors of the log-sum-exp's scores and of its slots' (twice the largest), the sums of V terms in
                 fp32 ((V / 16 + 64) 2^-24), and fp32 roundings of numbers as large as the scores and the log-sum-exp
  a gradient     every probability is off by u + delta of itself (delta: the error of its exponent, which is that of a score
                 and of the log-sum-exp), sums of n terms in fp32 by (n + 16) 2^-24 of the sum of magnitudes, fp16
                 probabilities below 2^-14 of the largest by 2^-25 * 2^-14 of that, the result by its own type's rounding
"""
from __future__ import annotations

import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U_P = {"f32": 2.0 ** -22, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
STEP_OUT = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


def weights(ids, logits, temperature):
    """(q, live): the teacher's weights over a row's slots, and whether the row has one with any weight."""
    live = ids >= 0
    if logits is None:
        q = live.double()
        return q, live.any(1)
    t = (logits.double() / temperature).masked_fill(~live, -math.inf)
    top = t.amax(1, keepdim=True)
    some = torch.isfinite(top[:, 0])
    e = torch.where(live & some[:, None], (t - torch.where(some[:, None], top, 0.0)).exp(), 0.0)
    return e / e.sum(1, keepdim=True).clamp_min(1e-300), some


def reference(h, w, ids, logits=None, temperature=1.0, scale=1.0, g=None):
    """Everything in 64 bits: loss, lse, mean, and with g grad_h, grad_w; beside them the bounds' ingredients."""
    ids = (ids if ids.dim() == 2 else ids[:, None]).long()
    s = scale / temperature
    q, some = weights(ids, logits, temperature)
    h, w = torch.where(some[:, None], h.double(), 0.0), w.double()
    z = h @ w.T * s
    lse = torch.logsumexp(z, 1)
    p = (z - lse[:, None]).exp()
    picked = z.gather(1, ids.clamp_min(0))
    loss = torch.where(q > 0, q * (q.clamp_min(1e-300).log() - picked + lse[:, None]), 0.0).sum(1)
    dense_q = torch.zeros_like(z).scatter_add_(1, ids.clamp_min(0), q)
    r = {"loss": torch.where(some, loss, 0.0), "lse": torch.where(some, lse, 0.0), "row_grad": torch.where(some[:, None], (p - dense_q) @ w * s, 0.0)}
    if g is not None:
        g = torch.where(some, g.double(), 0.0)
        d = g[:, None] * (p - dense_q) * s
        r["grad_h"], r["grad_w"] = d @ w, d.T @ h
    return r, dict(h=h, w=w, z=z, p=p, q=dense_q, s=s, some=some, lse=lse)


def bounds(dtype, x, g=None):
    h, w, s = x["h"].abs(), x["w"].abs(), x["s"]
    (T, D), V = h.shape, w.shape[0]
    a = (h @ w.T).amax(1) * s
    dz = (D + 4) * 2.0 ** -24 * a
    if dtype == "f32":
        dz = dz + 3 * 2.0 ** -22 * a + 2.0 ** -38 * D * h.amax() * w.amax() * s
    dlse = dz + (V / 16 + 64) * 2.0 ** -24 + 8 * 2.0 ** -24 * (x["lse"].abs() + x["z"].abs().amax(1))
    b = {"lse": dlse, "loss": 2 * dlse + 16 * 2.0 ** -24 * (x["lse"].abs() + x["z"].abs().amax(1) + 64)}
    u, lift = U_P[dtype], (0.0 if dtype == "bf16" else 2.0 ** -39)
    delta = (dz + dlse + 2.0 ** -20)[:, None]
    both = x["p"] + x["q"]
    b["row_grad"] = s * ((u + delta + (V + 80) * 2.0 ** -24) * (both @ w) + lift * 2 * w.sum(0))
    if g is not None:
        g = torch.where(x["some"], g.double().abs(), 0.0)
        b["grad_h"] = g[:, None] * (b["row_grad"] + s * 2.0 ** -24 * (both @ w))
        e = g[:, None] * both
        b["grad_w"] = s * ((u + (T + 80) * 2.0 ** -24) * (e.T @ h) + (e * delta).T @ h + lift * 2 * g.amax() * h.sum(0))
    return b


def check(got, ref, bound, dtype, what):
    """|got - ref| <= bound + the rounding of the output's own type."""
    own = U_OUT[dtype] * ref.abs() + STEP_OUT[dtype]
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    err = (got.double() - ref).abs()
    assert bool(torch.isfinite(got).all()), what + ": not finite"
    over = (err / (bound + own)).max().item() if err.numel() else 0.0
    assert over <= 1.0, "%s: %.3g times its bound (largest error %.3g)" % (what, over, err.max().item())
    return over


def inputs(op, dtype, T, V, D, K=0, seed=0, device="cuda:0", holes=True, spread=2.0):
    """Rows with a planted class, ids with holes, gradients of both signs; every row's IDs differ."""
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((V, D), generator=gen) * spread / math.sqrt(D)
    best = (torch.rand(T, generator=gen) ** 2 * V).long().clamp_(0, V - 1)
    h = torch.randn((T, D), generator=gen) + w[best] * (3.0 * torch.rand((T, 1), generator=gen))
    g = torch.rand(T, generator=gen) * 2.0 - 0.7
    if op == "xent":
        ids = torch.where(torch.rand(T, generator=gen) < (0.1 if holes else -1.0), -1, best).int()
        logits = None
    else:
        ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(T)]) if T else torch.zeros((0, K))
        if T:
            ids[:, 0] = torch.where((ids == best[:, None]).any(1), ids[:, 0], best)
        ids = torch.where(torch.rand((T, K), generator=gen) < (0.15 if holes else -1.0), -1, ids).int()
        logits = (torch.randn((T, K), generator=gen) * 3.0).to(DTYPES[dtype])
    to = lambda t: None if t is None else t.to(device)
    return to(h.to(DTYPES[dtype])), to(w.to(DTYPES[dtype])), to(ids), to(logits), to(g)

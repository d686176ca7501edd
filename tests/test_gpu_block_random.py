"""Seeded random sizes, types, activations, strides and offsets of the block's operators, each against its definition in 64 bits within
the bounds of block_bounds.py."""
import random

import pytest
import torch

import block_bounds as bb
import test_gpu_block_orthogonal as ortho

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _size(rng, most, grid=None):
    n = int(round(2 ** rng.uniform(0, most)))
    return n if grid is None or rng.random() < 0.5 else -(-n // grid) * grid


def _rows(rng, t):
    """The same rows somewhere in a wider buffer, in half of the cases."""
    if rng.random() < 0.5:
        return t
    before, behind = rng.choice([(0, 8), (3, 2), (8, 0), (1, 0)])
    wide = torch.full((t.shape[0], before + t.shape[1] + behind), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, before:before + t.shape[1]] = t
    return wide[:, before:before + t.shape[1]]


@pytest.mark.parametrize("seed", range(40))
def test_gated(seed):
    from paper_2511_13645_amd import binding as fsa
    rng = random.Random(seed)
    dtype, act = rng.choice(TYPES), rng.choice(["silu", "gelu", "relu"])
    t, d, h, o = _size(rng, 12.5), _size(rng, 10, 8), _size(rng, 10.5, 8), _size(rng, 9, 8)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    x, wg, wu, wd, gy = (_rows(rng, v.to(dtype)) for v in (n(t, d), n(h, d) * 1.5 * d ** -0.5, n(h, d) * 1.5 * d ** -0.5, n(o, h) * h ** -0.5,
                                                            n(t, o) * 2.0 ** rng.randint(-12, 4)))
    want = bb.gated(x, wg, wu, wd, gy, act, dtype)
    kept = None
    if rng.random() < 0.5:
        y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act, emit_kept=True)
    else:
        y = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act)
    bb.check("y", y, *want["y"])
    wanted = [rng.random() < 0.8 for _ in range(4)]
    for name, w, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), wanted, fsa.fsa_gated_bwd(gy, x, wg, wu, wd, kept, activation=act, want=wanted)):
        assert (g is not None) == w
        if w:
            bb.check(name, g, *want[name])


@pytest.mark.parametrize("seed", range(30))
def test_norm(seed):
    from paper_2511_13645_amd import binding as fsa
    rng = random.Random(1000 + seed)
    dtype, wdtype = rng.choice(TYPES), rng.choice(TYPES)
    t, d = _size(rng, 12), _size(rng, 14, 8)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    x, r = _rows(rng, n(t, d).to(dtype)), _rows(rng, n(t, d).to(dtype)) if rng.random() < 0.6 else None
    w, gy, gs = n(d).to(wdtype), n(t, d).to(dtype), n(t, d).to(dtype) if rng.random() < 0.5 else None
    want = bb.norm(x, r, w, gy, gs, 1e-6, dtype)
    y, s = fsa.fsa_norm_fwd(x, w, r, 1e-6)
    bb.check("y", y, *want["y"])
    if r is not None:
        bb.check("s", s, *want["s"])
    gx, gw = fsa.fsa_norm_bwd(gy, gs, x if r is None else s, w, 1e-6)
    bb.check("grad_x", gx, *want["grad_x"])
    bb.check("grad_weight", gw, *want["grad_weight"])


@pytest.mark.parametrize("seed", range(25))
def test_orthogonal(seed):
    from paper_2511_13645_amd import binding as fsa
    rng = random.Random(2000 + seed)
    dtype, steps = rng.choice(TYPES), rng.randint(1, 5)
    b, m, n = rng.choice([None, 1, 2, 5]), _size(rng, 10, 8), _size(rng, 10, 8)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    g = (torch.randn(((b,) if b else ()) + (m, n + 5), generator=gen, device=DEV) * 2.0 ** rng.randint(-8, 3)).to(dtype)
    g = g[..., :n] if rng.random() < 0.5 else g[..., :n].contiguous()
    got = fsa.fsa_orthogonalize(g, ortho.ABC, steps)
    assert got.shape == g.shape and got.dtype == dtype
    ortho._check(got, ortho._reference(g, [ortho.ABC] * steps), steps, dtype)

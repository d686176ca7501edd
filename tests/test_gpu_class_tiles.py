"""Class losses where every workgroup streams several tiles: the rotation of tiles in LDS, the running reference from one tile to
the next, slots asked for tiles ahead, tables laid out first, and offsets beyond 32 bits, against the definition in 64 bits."""
import math

import pytest
import torch

from class_bounds import bounds
from class_tiles import BOTH, FEW_CLASSES, FEW_ROWS, WIDE
from class_util import DTYPES, check, inputs, reference

pytestmark = pytest.mark.gpu


def compare(dtype, h, w, ids, logits, g, temperature=1.0, scale=1.0):
    from paper_2511_13645_amd import binding as fsa
    ref, x = reference(h, w, ids, logits, temperature, scale, g)
    lim = bounds(dtype, x, g)
    if logits is None:
        alone = fsa.fsa_xent_fwd(h, w, ids, scale)
        f = fsa.fsa_xent_fwd(h, w, ids, scale, emit_row_grad=True)
        b = fsa.fsa_xent_bwd(g, h, w, ids, f[1], f[2], scale)
    else:
        alone = fsa.fsa_distill_fwd(h, w, ids, logits, temperature, scale)
        f = fsa.fsa_distill_fwd(h, w, ids, logits, temperature, scale, emit_row_grad=True)
        b = fsa.fsa_distill_bwd(g, h, w, ids, logits, f[1], f[2], temperature, scale)
    for name, got, d in (("loss", f[0], "f32"), ("lse", f[1], "f32"), ("row_grad", f[2], "f32"), ("grad_h", b[0], dtype), ("grad_w", b[1], dtype)):
        check(got, ref[name], lim[name], d, name)
    check(alone[0], ref["loss"], lim["loss"], "f32", "loss alone")
    check(alone[1], ref["lse"], lim["lse"], "f32", "lse alone")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", BOTH + FEW_ROWS + FEW_CLASSES + WIDE)
def test_cross_entropy(dtype, T, V, D):
    h, w, ids, _, g = inputs("xent", dtype, T, V, D, seed=T + D)
    compare(dtype, h, w, ids, None, g, scale=0.75)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", BOTH[::2] + FEW_ROWS[1::2] + FEW_CLASSES[1::2] + WIDE[::2])
@pytest.mark.parametrize("K", [2, 5, 17])
def test_distillation(dtype, T, V, D, K):
    h, w, ids, logits, g = inputs("distill", dtype, T, V, D, K, seed=T + D + K)
    compare(dtype, h, w, ids, logits, g, temperature=2.0, scale=1.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [BOTH[2], BOTH[5], FEW_ROWS[1], FEW_ROWS[4], WIDE[0], WIDE[2]])
def test_the_running_maximum_moves(dtype, T, V, D):
    """Classes in the order of how much every row likes them: each tile has a larger maximum than the one before, and the other
    way round, so that the reference moves in every tile or in the first alone."""
    h, w, ids, _, g = inputs("xent", dtype, T, V, D, seed=V + D, spread=6.0)
    h[:, 0] = 4.0
    for end in (1.0, -1.0):
        w[:, 0] = (end * torch.linspace(-6.0, 6.0, V, device=w.device)).to(w.dtype)
        compare(dtype, h, w, ids, None, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [BOTH[2], BOTH[3], FEW_ROWS[2], WIDE[0], WIDE[1]])
def test_strides(dtype, T, V, D):
    """Rows apart, off the 16-byte grid and on it."""
    h, w, ids, _, g = inputs("xent", dtype, T, V, D, seed=7)
    for off, more in ((1, 5), (8, 24)):
        big_h = torch.full((T + 1, D + more), math.nan, dtype=h.dtype, device=h.device)
        big_w = torch.full((V + 1, D + more), math.nan, dtype=h.dtype, device=h.device)
        vh, vw = big_h[1:, off:off + D], big_w[1:, off:off + D]
        vh.copy_(h)
        vw.copy_(w)
        compare(dtype, vh, vw, ids, None, g)


@pytest.mark.parametrize("V,D,T", [(17_000_000, 128, 300), (22_000_000, 100, 20), (2_200_000, 1000, 40)])
def test_fp32_tables_beyond_32_bit_offsets(V, D, T):
    """fp32 tables of more than 2^31 elements and their planes: the first and last classes and some between.  A sum of V terms over
    a hundred workgroups and more is right to V / 200 roundings."""
    from paper_2511_13645_amd import binding as fsa
    assert 2 ** 31 // D + 1 < V, "the class at the offset that 32 bits end at is one of the table's"
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    w = torch.empty((V, D), device="cuda:0").normal_(0, 1.0 / math.sqrt(D), generator=gen)
    h = torch.randn((T, D), generator=gen, device="cuda:0")
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda:0").int()
    ids[:5] = torch.tensor([0, V - 1, V // 2, 2 ** 31 // D, -1], dtype=torch.int32)
    g = torch.rand(T, generator=gen, device="cuda:0") - 0.4
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    alone = fsa.fsa_xent_fwd(h, w, ids)
    gh, gw = fsa.fsa_xent_bwd(g, h, w, ids, lse, rg)
    total, mean = torch.zeros(T, dtype=torch.float64, device="cuda:0"), torch.zeros((T, D), dtype=torch.float64, device="cuda:0")
    step = 1 << 18
    for a in range(0, V, step):
        e = (h.double() @ w[a:a + step].double().T).exp()
        total += e.sum(1)
        mean += e @ w[a:a + step].double()
    live, y = ids >= 0, ids.clamp(min=0).long()
    off = V / 200 * 2.0 ** -24 + 1e-5
    z = (h.double() * w[y].double()).sum(1)
    for x in (lse, alone[1]):
        assert float((x - total.log())[live].abs().max()) < off
    for x in (loss, alone[0]):
        assert float((x - (total.log() - z))[live].abs().max()) < off
    row = g.double()[:, None] * (mean / total[:, None] - w[y].double())
    check(gh[live], row[live], (off * g.double().abs()[:, None] * (w[y].double().abs() + 1e-2))[live], "f32", "grad_h")
    rows = torch.cat([y[live], torch.tensor([1, V - 2, 2 ** 31 // D + 1], device="cuda:0")])
    p = (h.double() @ w[rows].double().T - total.log()[:, None]).exp()
    d = (p - (rows[None, :] == ids[:, None]).double()) * torch.where(live, g.double(), 0.0)[:, None]
    floor = 2.0 ** -38 * T * float((g.abs() * h.abs().amax(1)).max())
    check(gw[rows], d.T @ h.double(), 2 * off * (d.abs().T @ h.double().abs()) + floor, "f32", "grad_w")

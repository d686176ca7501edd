"""Gradients of rows that have learned their class, and of students that agree with their teacher: p and q nearly cancel there,
and what is left of them has to be right."""
import math

import pytest
import torch

from class_bounds import bounds
from class_util import DTYPES, check, reference

pytestmark = pytest.mark.gpu


def learned(dtype, T, V, D, seed):
    """Rows h = c * (their class's row) + a little, all of them numbers of 7 bits whose products and sums are exact in fp32: p of
    the own class is from about one half up to 1 - 1e-7."""
    gen = torch.Generator().manual_seed(seed)
    scale = 2.0 ** -round(math.log2(D / 8))
    w = torch.randint(-2, 3, (V, D), generator=gen) / 2
    best = torch.randint(0, V, (T,), generator=gen)
    c = torch.randint(12, 49, (T, 1), generator=gen) / 8
    h = c * w[best] + torch.randint(-1, 2, (T, D), generator=gen) / 8
    g = (0.5 + torch.rand(T, generator=gen)) * torch.where(torch.rand(T, generator=gen) < 0.2, -1.0, 1.0)
    to = lambda t: t.to(DTYPES[dtype]).cuda()
    return to(h), to(w), best.int().cuda(), g.cuda(), scale


def gradients(dtype, h, w, ids, logits, g, scale):
    from paper_2511_13645_amd import binding as fsa
    if logits is None:
        loss, lse, row_grad = fsa.fsa_xent_fwd(h, w, ids, scale, emit_row_grad=True)
        grad_h, grad_w = fsa.fsa_xent_bwd(g, h, w, ids, lse, row_grad, scale)
    else:
        loss, lse, row_grad = fsa.fsa_distill_fwd(h, w, ids, logits, 1.0, scale, emit_row_grad=True)
        grad_h, grad_w = fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, 1.0, scale)
    ref, x = reference(h, w, ids, logits, 1.0, scale, g)
    lim = bounds(dtype, x, g, exact=True)
    return (("loss", loss, ref["loss"], lim["loss"], "f32"), ("lse", lse, ref["lse"], lim["lse"], "f32"),
            ("row_grad", row_grad, ref["row_grad"], lim["row_grad"], "f32"), ("grad_h", grad_h, ref["grad_h"], lim["grad_h"], dtype),
            ("grad_w", grad_w, ref["grad_w"], lim["grad_w"], dtype))


# few rows and classes; rows that wait for a second tile of classes and of rows; the widths around where rows become long
SIZES = [(3, 50, 64), (40, 47, 128), (64, 500, 256), (64, 500, 320), (33, 130, 602), (200, 300, 96), (2100, 9000, 128),
         (1100, 5000, 64), (700, 9000, 384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("name", ["row_grad", "grad_w"])
def test_cross_entropy_of_learned_rows(dtype, T, V, D, name):
    h, w, ids, g, scale = learned(dtype, T, V, D, T + D)
    for n, got, ref, lim, d in gradients(dtype, h, w, ids, None, g, scale):
        if n in (name, "loss", "lse", "grad_h" if name == "row_grad" else name):
            check(got, ref, lim, d, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("K", [3, 40])
@pytest.mark.parametrize("name", ["row_grad", "grad_w"])
def test_students_that_agree_with_their_teacher(dtype, T, V, D, K, name):
    """The teacher's logits are the student's own scores of its K best classes; a few slots empty, a few named twice."""
    h, w, best, g, scale = learned(dtype, T, V, D, T + D + K)
    z = torch.cat([h[a:a + 256].double() @ w.double().T for a in range(0, T, 256)]) * scale
    top, ids = z.topk(K, 1)
    logits, ids = top.float(), ids.int()
    gen = torch.Generator().manual_seed(K)
    order = torch.argsort(torch.rand(ids.shape, generator=gen), 1).cuda()
    ids, logits = ids.gather(1, order), logits.gather(1, order).contiguous()
    ids[torch.rand(ids.shape, generator=gen).cuda() < 0.05] = -1
    ids[::3, 1] = ids[::3, 0]
    ids = ids.contiguous()
    for n, got, ref, lim, d in gradients(dtype, h, w, ids, logits, g, scale):
        if n in (name, "loss", "lse", "grad_h" if name == "row_grad" else name):
            check(got, ref, lim, d, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 300])
def test_many_slots_that_name_one_class(dtype, D):
    """Weights of slots that name the same class are summed in slot order: the same bits every time, and the right ones."""
    from paper_2511_13645_amd import binding as fsa
    h, w, best, g, scale = learned(dtype, 70, 90, D, 5)
    gen = torch.Generator().manual_seed(1)
    ids = torch.randint(0, 90, (70, 3), generator=gen).cuda()[:, torch.randint(0, 3, (40,), generator=gen).cuda()].int().contiguous()
    ids[:, ::7] = best[:, None]
    logits = torch.randn((70, 40), generator=gen).cuda()
    for n, got, ref, lim, d in gradients(dtype, h, w, ids, logits, g, scale):
        if n in ("grad_h", "grad_w"):
            check(got, ref, lim, d, n)
    loss, lse, row_grad = fsa.fsa_distill_fwd(h, w, ids, logits, 1.0, scale, emit_row_grad=True)
    first = fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, 1.0, scale)
    for _ in range(5):
        again = fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, 1.0, scale)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_losses_of_learned_rows(dtype, T, V, D):
    """Where gradients are wanted, a loss of 1e-7 is right to a share of itself: that of a sum of V terms and of 2^20."""
    from paper_2511_13645_amd import binding as fsa
    h, w, ids, g, scale = learned(dtype, T, V, D, T + D + 1)
    ref, x = reference(h, w, ids, None, 1.0, scale, g)
    loss = fsa.fsa_xent_fwd(h, w, ids, scale, emit_row_grad=True)[0]
    share = (V / 16 + 64 + 8 * x["z"].abs().amax(1)) * 2.0 ** -24 + 2.0 ** -20
    check(loss, ref["loss"], share * ref["loss"] + 2.0 ** -48, "f32", "loss")

"""Class losses on tables whose elements are far apart in size: masks in a column of biases, very small and very large tables,
teacher logits at the end of their type."""
import math

import pytest
import torch

from class_bounds import bounds
from class_util import check, inputs, reference

pytestmark = pytest.mark.gpu


def compare(dtype, h, w, ids, logits=None, g=None, temperature=1.0, scale=1.0, grads=True):
    from paper_2511_13645_amd import binding as fsa
    ref, x = reference(h, w, ids, logits, temperature, scale, g)
    lim = bounds(dtype, x, g)
    fwd = (lambda **kw: fsa.fsa_xent_fwd(h, w, ids, scale, **kw)) if logits is None else (
        lambda **kw: fsa.fsa_distill_fwd(h, w, ids, logits, temperature, scale, **kw))
    loss, lse, row_grad = fwd(emit_row_grad=True)
    alone, lse_alone, _ = fwd()
    for n, got, name in (("loss", loss, "loss"), ("lse", lse, "lse"), ("loss alone", alone, "loss"), ("lse alone", lse_alone, "lse")):
        check(got, ref[name], lim[name], "f32", n)
    if not grads:
        return
    check(row_grad, ref["row_grad"], lim["row_grad"], "f32", "row_grad")
    if logits is None:
        grad_h, grad_w = fsa.fsa_xent_bwd(g, h, w, ids, lse, row_grad, scale)
    else:
        grad_h, grad_w = fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, temperature, scale)
    check(grad_h, ref["grad_h"], lim["grad_h"], dtype, "grad_h")
    check(grad_w, ref["grad_w"], lim["grad_w"], dtype, "grad_w")


# one workgroup's waves beside each other or after each other, tables laid out first (wide ones always, narrow ones of many
# workgroups) and read as they are
SIZES = [(5, 3000, 40), (40, 47, 128), (70, 900, 200), (300, 3000, 100), (600, 9000, 128), (5, 2000, 300), (70, 900, 602), (200, 3000, 384)]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("mask", [-1e6, -1e9, -1e12, torch.finfo(torch.float32).min])
def test_masked_classes(T, V, D, mask):
    """A bias as a column of ones in h and a column of w, which at masked classes is a large negative number: those get no
    probability, and the others keep theirs."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=T)
    h[:, -1] = 1.0
    masked = torch.zeros(V, dtype=torch.bool, device=h.device)
    masked[::3] = True
    w[masked, -1] = mask
    ids[torch.isin(ids, masked.nonzero()[:, 0])] += 1                       # no row asks for a masked class
    compare("f32", h, w, ids.clamp(max=V - 2 if masked[V - 1] else V - 1), g=g, scale=0.75)


@pytest.mark.parametrize("T,V,D", SIZES)
def test_a_masked_class_is_asked_for(T, V, D):
    """A target or a teacher's class that is masked: its loss is what the mask says, its gradients pull."""
    h, w, ids, logits, g = inputs("distill", "f32", T, V, D, 5, seed=D)
    h[:, -1] = 1.0
    w[::4, -1] = -1e5
    compare("f32", h, w, ids, logits, g)


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("size", [1e12, 1e25])
def test_rows_that_diverge(T, V, D, size):
    """A row of h far larger than the others: its own scores are lost to its softmax, everybody else's losses are not."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=V)
    h[3] *= size
    compare("f32", h, w, ids, g=g)


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("size", [1e12, 1e25])
def test_classes_that_diverge(T, V, D, size):
    """A class far larger than the others takes the rows on its side and leaves the others as they are."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=V + 1)
    w[V // 2] *= size
    compare("f32", h, w, ids, g=g)


@pytest.mark.parametrize("T,V,D", SIZES)
def test_rows_and_classes_of_all_sizes(T, V, D):
    """Rows and classes 2^-20 to 1 times as large, and all of h as much larger as all of w is smaller."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=D + 1)
    gen = torch.Generator().manual_seed(3)
    rows = torch.exp2(torch.randint(-20, 1, (T, 1), generator=gen).float()).cuda()
    classes = torch.exp2(torch.randint(-20, 1, (V, 1), generator=gen).float()).cuda()
    compare("f32", h * rows, w * classes, ids, g=g / rows[:, 0])
    for k in (-40, 40):
        compare("f32", h * 2.0 ** k, w * 2.0 ** -k, ids, g=g)


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("size", [1e-15, 1e-19, 1e-24, 1e-37])
def test_very_small_tables(T, V, D, size):
    """Scores of nothing: every class is as likely, the loss is log V."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=9)
    compare("f32", h * size, w * size, ids, g=g, grads=size > 1e-30)


@pytest.mark.parametrize("D", [64, 300])
def test_scores_far_below_zero(D, dtype="f32"):
    """Every score of a row far below -1e30: the largest of them is the log-sum-exp all the same."""
    from paper_2511_13645_amd import binding as fsa
    T, V = 40, 70
    h, w, ids, _, _ = inputs("xent", dtype, T, V, D, holes=False)
    h.zero_()
    w.zero_()
    h[:, 0] = 2.0 ** 53
    w[:, 0] = -(2.0 ** 53) * (1 + torch.arange(V, device=h.device) % 2).to(w.dtype)
    want = -(2.0 ** 106)                                 # of half of the classes; the others have twice that
    ids = (ids // 2 * 2).contiguous()
    loss, lse, row_grad = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    alone = fsa.fsa_xent_fwd(h, w, ids)
    for got in (lse, alone[1]):
        assert float((got.double() / want - 1).abs().max()) < 2.0 ** -20
    for got in (loss, alone[0]):
        assert float(got.double().abs().max()) <= 2.0 ** -20 * abs(want)
    assert bool(torch.isfinite(row_grad).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 300])
@pytest.mark.parametrize("temperature", [0.25, 0.5, 1.0, 3.0])
def test_teacher_logits_at_the_end_of_their_type(dtype, D, temperature):
    """Logits that the temperature would take out of range: only their differences count.  A row of nothing but the lowest
    number is one of equal weights, and one of nothing but the highest too."""
    h, w, ids, logits, g = inputs("distill", dtype, 12, 90, D, 8, holes=False)
    logits = logits.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    ends = torch.finfo(logits.dtype)
    logits[0] = ends.min
    logits[1] = ends.max
    logits[2, 2:] = ends.min
    logits[3, :3] = ends.max
    logits[4, ::2] = -math.inf
    compare(dtype, h, w, ids, logits, g, temperature)


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("size", [1e-6, 1.0, 1e6])
def test_columns_of_zeros(T, V, D, size):
    """Seven of eight columns zero, whichever of them they are, in tables of any size."""
    for keep in range(8):
        h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=keep)
        drop = torch.arange(D, device=h.device) % 8 != keep
        h[:, drop], w[:, drop] = 0.0, 0.0
        compare("f32", h * size, w / size, ids, g=g)

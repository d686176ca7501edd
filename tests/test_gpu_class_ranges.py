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
@pytest.mark.parametrize("size", [1e-15, 1e-19, 1e-24, 1e-37])
def test_very_small_tables(T, V, D, size):
    """Scores of nothing: every class is as likely, the loss is log V."""
    h, w, ids, _, g = inputs("xent", "f32", T, V, D, seed=9)
    compare("f32", h * size, w * size, ids, g=g, grads=size > 1e-30)


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

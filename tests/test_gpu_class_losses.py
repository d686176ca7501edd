"""Softmax cross entropy and distillation over many classes against their definition in 64 bits: every type, rows from
none to several tiles, classes from one up, odd depths, holes and rows without a slot, strides, gradients alone."""
import math

import pytest
import torch

from class_util import DTYPES, bounds, check, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fsa():
    from paper_2511_13645_amd import binding
    binding.lib()
    return binding


def forward(fsa, op, h, w, ids, logits, temperature, scale, **kw):
    if op == "xent":
        return fsa.fsa_xent_fwd(h, w, ids, scale, **kw)
    return fsa.fsa_distill_fwd(h, w, ids, logits, temperature, scale, **kw)


def backward(fsa, op, g, h, w, ids, logits, lse, row_grad, temperature, scale, **kw):
    if op == "xent":
        return fsa.fsa_xent_bwd(g, h, w, ids, lse, row_grad, scale, **kw)
    return fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, temperature, scale, **kw)


def compare(fsa, op, dtype, h, w, ids, logits, g, temperature=1.0, scale=1.0):
    """Forward and backward against the definition; returns what they gave."""
    ref, x = reference(h, w, ids, logits, temperature, scale, g)
    lim = bounds(dtype, x, g)
    loss, lse, row_grad = forward(fsa, op, h, w, ids, logits, temperature, scale, emit_row_grad=True)
    alone, lse_alone, none = forward(fsa, op, h, w, ids, logits, temperature, scale)
    assert none is None
    grad_h, grad_w = backward(fsa, op, g, h, w, ids, logits, lse, row_grad, temperature, scale)
    assert grad_h.dtype == h.dtype and grad_w.dtype == w.dtype
    for name, got, d in (("loss", loss, "f32"), ("lse", lse, "f32"), ("row_grad", row_grad, "f32"), ("grad_h", grad_h, dtype),
                         ("grad_w", grad_w, dtype)):
        check(got, ref[name], lim[name], d, name)
    check(alone, ref["loss"], lim["loss"], "f32", "loss alone")
    check(lse_alone, ref["lse"], lim["lse"], "f32", "lse alone")
    return loss, lse, row_grad, grad_h, grad_w


SIZES = [(1, 1, 1), (1, 47, 128), (2, 33, 3), (5, 1000, 64), (31, 64, 100), (32, 32, 32), (33, 129, 65), (64, 31, 128),
         (65, 4097, 37), (127, 500, 256), (128, 2, 255), (129, 96, 129), (200, 3001, 96), (300, 65, 200), (513, 129, 16),
         (1, 1, 257), (33, 700, 602), (70, 95, 384), (65, 33, 1024), (129, 257, 640), (40, 1500, 385)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_cross_entropy(fsa, dtype, T, V, D):
    h, w, ids, _, g = inputs("xent", dtype, T, V, D, seed=T + V + D)
    compare(fsa, "xent", dtype, h, w, ids, None, g, scale=0.75)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,K", [(1, 1, 8, 1), (3, 70, 20, 64), (40, 64, 64, 64), (65, 1000, 100, 10), (130, 2049, 128, 33),
                                     (257, 200, 250, 5), (1, 5000, 128, 17), (70, 300, 602, 50), (33, 64, 300, 64), (65, 40, 1001, 3)])
def test_distillation(fsa, dtype, T, V, D, K):
    h, w, ids, logits, g = inputs("distill", dtype, T, V, D, K, seed=T + V + K)
    compare(fsa, "distill", dtype, h, w, ids, logits, g, temperature=2.0, scale=1.5)

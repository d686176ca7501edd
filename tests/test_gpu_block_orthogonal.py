"""Orthogonalised matrices against the definition in 64 bits.

Tolerance: a step's products are sums of up to n fp32 products of elements held to 2^-24, so that a step is off by about
(8 + sqrt n) 2^-24 of what it adds up (roundings of either sign), (|a| + |b| + |c|) |X|_F; later steps multiply an error by no more than the
polynomial's steepest slope, 4 over singular values up to 1.21.  Then half a step of the type."""
import math

import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ABC = (3.4445, -4.7750, 2.0315)


def _reference(g, coefficients, eps=1e-7):
    x = g.double()
    x = x / (torch.linalg.vector_norm(x, dim=(-2, -1), keepdim=True) + eps)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT.contiguous()
    for a, b, c in coefficients:
        gram = x @ x.mT.contiguous()
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.mT.contiguous() if tall else x


def _check(got, want, steps, dtype):
    m, n = sorted(want.shape[-2:])
    for x, y in zip(got.reshape(-1, *want.shape[-2:]), want.reshape(-1, *want.shape[-2:])):
        size = y.norm().item()
        off = (x.double() - y).norm().item()
        each = (8 + math.sqrt(n)) * bb.V * sum(map(abs, ABC)) * max(1.0, size)
        assert off <= each * sum(4.0 ** i for i in range(steps)) + bb.HALF_STEP[dtype] * size + bb.FLOOR[dtype] * math.sqrt(m * n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,m,n", [(None, 1, 1), (None, 1, 50), (None, 50, 1), (None, 3, 5), (None, 16, 16), (None, 64, 64), (None, 65, 63),
                                   (None, 100, 47), (None, 128, 512), (None, 512, 128), (None, 130, 1030), (None, 602, 300), (1, 40, 60),
                                   (3, 33, 70), (3, 70, 33), (7, 128, 128)])
def test_one_step_and_five(b, m, n, dtype):
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(m * n)
    g = (torch.randn(((b,) if b else ()) + (m, n), generator=gen, device=DEV) * 1e-2).to(dtype)
    for steps in (1, 2, 5):
        got = fsa.fsa_orthogonalize(g, ABC, steps)
        assert got.shape == g.shape and got.dtype == dtype
        _check(got, _reference(g, [ABC] * steps), steps, dtype)


@pytest.mark.parametrize("edge", [130, 1100])
def test_wide_tiles_and_many_of_them(edge):
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(edge)
    g = torch.randn((70 if edge < 200 else 4, edge, edge + 60), generator=gen, device=DEV)
    _check(fsa.fsa_orthogonalize(g, ABC, 2), _reference(g, [ABC] * 2), 2, torch.float32)


def test_coefficients_of_every_step_scale_and_a_matrix_that_is_nearly_orthogonal():
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(0)
    g = torch.randn((96, 160), generator=gen, device=DEV)
    triples = [(3.4445, -4.775, 2.0315)] * 4 + [(1.875, -1.25, 0.375)] * 4
    x = fsa.fsa_orthogonalize(g, triples)
    _check(x, _reference(g, triples), 8, torch.float32)
    assert (x @ x.T - torch.eye(96, device=DEV)).abs().max().item() < 1e-2
    assert torch.equal(fsa.fsa_orthogonalize(g, triples, scale=0.25), x * 0.25)


@pytest.mark.parametrize("unit", [1e-30, 1e-12, 1e12, 1e30])
def test_matrices_of_any_magnitude(unit):
    from paper_2511_13645_amd import binding as fsa
    g = torch.randn((48, 80), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) * unit
    _check(fsa.fsa_orthogonalize(g, ABC, 3, eps=0.0), _reference(g, [ABC] * 3, 0.0), 3, torch.float32)


def test_zeros_and_what_is_not_finite_stay_by_themselves():
    from paper_2511_13645_amd import binding as fsa
    g = torch.randn((4, 30, 40), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    whole = fsa.fsa_orthogonalize(g)
    g[1] = 0.0
    g[2, 3, 4] = float("inf")
    for eps in (0.0, 1e-7):
        x = fsa.fsa_orthogonalize(g, eps=eps)
        assert torch.equal(x[1], torch.zeros_like(x[1])) and x[2].isnan().all()
        if eps:
            assert torch.equal(x[0], whole[0]) and torch.equal(x[3], whole[3])
    assert fsa.fsa_orthogonalize(g[:0]).shape == (0, 30, 40)


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_matrices(dtype):
    from paper_2511_13645_amd import binding as fsa
    room = torch.randn((3, 50, 90), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dtype)
    view = room[:, 7:47, 3:64]
    assert torch.equal(fsa.fsa_orthogonalize(view), fsa.fsa_orthogonalize(view.contiguous()))
    assert torch.equal(fsa.fsa_orthogonalize(view[1]), fsa.fsa_orthogonalize(view[1].contiguous()))
    one = room[:1, :40].expand(3, 40, 90)                    # one matrix three times
    assert torch.equal(fsa.fsa_orthogonalize(one)[2], fsa.fsa_orthogonalize(one[0]))

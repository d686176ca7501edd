"""Orthogonalised matrices of elements at the ends of fp32, where neither their norm nor what it is divided into is a number of 32
bits."""
import pytest
import torch

import block_bounds as bb
import test_gpu_block_orthogonal as ortho

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _matrix(m, n):
    """Elements of [1, 2) with either sign: powers of two of them are exact as long as they are normal numbers."""
    gen = torch.Generator(device=DEV).manual_seed(m)
    u = 1.0 + torch.rand((m, n), generator=gen, device=DEV)
    return u * (2.0 * (torch.rand((m, n), generator=gen, device=DEV) < 0.5) - 1.0)


@pytest.mark.parametrize("m,n", [(48, 80), (200, 60), (1, 1), (300, 301)])
@pytest.mark.parametrize("power", [-126, -122, -100, 100, 120, 126])
def test_a_power_of_two_changes_nothing(m, n, power):
    from paper_2511_13645_amd import binding as fsa
    g = _matrix(m, n)
    want = fsa.fsa_orthogonalize(g, ortho.ABC, 3, eps=0.0)
    ortho._check(want, ortho._reference(g, [ortho.ABC] * 3, 0.0), 3, torch.float32)
    assert torch.equal(fsa.fsa_orthogonalize(torch.ldexp(g, torch.tensor(power, device=DEV)), ortho.ABC, 3, eps=0.0), want)


def test_subnormal_elements():
    from paper_2511_13645_amd import binding as fsa
    g = torch.ldexp(_matrix(40, 70).double(), torch.tensor(-135, device=DEV)).float()
    assert 0.0 < g.abs().max().item() < 2.0 ** -126
    ortho._check(fsa.fsa_orthogonalize(g, ortho.ABC, 3, eps=0.0), ortho._reference(g, [ortho.ABC] * 3, 0.0), 3, torch.float32)


def test_elements_far_below_the_largest():
    # one step of a x alone: what comes back is what was held, 23 bits down to 2^-15 of the norm and 2^-38 of it below
    from paper_2511_13645_amd import binding as fsa
    g = _matrix(8, 64)
    g[1:] *= torch.logspace(0, -12, 7, device=DEV)[:, None]
    x = g.double() / g.double().norm()
    off = (fsa.fsa_orthogonalize(g, [(1.0, 0.0, 0.0)], eps=0.0).double() - x).abs()
    # (and fp32's own rounding of what is divided and of what comes back)
    assert (off <= x.abs() * 2.0 ** -23 + 3 * bb.V * x.abs() + 2.0 ** -38).all()

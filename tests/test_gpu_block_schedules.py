"""Orthogonalised matrices by steps with coefficients of their own, steep ones among them, against the definition in 64 bits.

Tolerance: as in test_gpu_block_orthogonal.py, a step is off by (8 + sqrt n) 2^-24 of what it adds up, (|a| + |b| s^2 + |c| s^4) |X|_F with s its
largest singular value, and later steps multiply that by no more than their polynomial's steepest slope up to theirs."""
import math

import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _reference(g, triples):
    """The result and its bound."""
    x = g.double()
    x = x / x.norm()
    if x.shape[0] > x.shape[1]:
        r, bound = _reference(g.mT.contiguous(), triples)
        return r.mT.contiguous(), bound
    off = 0.0
    for a, b, c in triples:
        s = torch.linalg.matrix_norm(x, 2).item()
        t = torch.linspace(0, s, 10_001, dtype=torch.float64) ** 2
        slope = (a + 3 * b * t + 5 * c * t * t).abs().max().item() * 1.001
        off = off * slope + (8 + math.sqrt(x.shape[1])) * bb.V * (abs(a) + abs(b) * s ** 2 + abs(c) * s ** 4) * x.norm().item()
        gram = x @ x.mT.contiguous()
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x, off


STEEP = (8.0, -23.0, 16.5)
SCHEDULES = {
    "steep first steps": [STEEP, (1.766, -0.644, 0.072), (3.4445, -4.775, 2.0315)],
    "steep alone": [STEEP],
    "larger and back": [(16.0, 16.0, 16.0), (0.02, 0.0, 0.0)],
    "a large A": [(5.0, 0.0, 0.0), (0.3, 0.01, -0.001)],
    "a large P": [(16.0, -15.5, 16.0), (0.05, 0.0, 0.0)],
    "scaled up": [(16.0, 0.0, 0.0), (16.0, 0.0, 0.0), (2.0 ** -8, 0.0, 0.0)],
}


@pytest.mark.parametrize("name", sorted(SCHEDULES))
@pytest.mark.parametrize("m,n", [(1, 40), (96, 160), (160, 96), (200, 1500)])
def test_schedules(m, n, name):
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(m)
    # few strong directions, the first with nearly all of the norm, so that a singular value is near one
    g = torch.randn((m, n), generator=gen, device=DEV)
    g += 30.0 * torch.randn((m, 1), generator=gen, device=DEV) * torch.randn((1, n), generator=gen, device=DEV)
    want, bound = _reference(g, SCHEDULES[name])
    got = fsa.fsa_orthogonalize(g, SCHEDULES[name], eps=0.0)
    assert want.isfinite().all()
    assert (got.double() - want).norm().item() <= bound + bb.V * want.norm().item()


def test_what_is_taken():
    from paper_2511_13645_amd import binding as fsa
    g = torch.ones((4, 4), device=DEV)
    with pytest.raises(fsa.FsaError, match="singular values"):
        fsa.fsa_orthogonalize(g, [(8.0, 23.0, 16.5)])

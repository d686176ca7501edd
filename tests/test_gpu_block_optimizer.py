"""Orthogonalised momentum: parameters may lie in memory as they like."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


@pytest.mark.parametrize("count", [1, 2])
@pytest.mark.parametrize("nesterov", [True, False])
def test_parameters_whose_columns_are_contiguous(count, nesterov):
    from paper_2511_13645_amd.orthogonal import OrthogonalMomentum
    results = []
    for turned in (False, True):
        rows = [_normal(30, 50, seed=i) for i in range(count)]
        params = [torch.nn.Parameter(r.t().contiguous().t() if turned else r.clone()) for r in rows]
        assert all((p.stride(0) == 1) == turned for p in params)
        opt = OrthogonalMomentum(params, 0.1, nesterov=nesterov)
        for step in range(3):
            for i, p in enumerate(params):
                p.grad = torch.empty_like(p).copy_(_normal(30, 50, seed=10 * step + i))
                assert p.grad.stride() == p.stride()
            opt.step()
        results.append([p.detach().clone() for p in params])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_gradients_that_autograd_makes_of_them():
    from paper_2511_13645_amd.orthogonal import OrthogonalMomentum
    w = torch.nn.Parameter(_normal(50, 30).t())
    opt = OrthogonalMomentum([w], 0.1)
    before = w.detach().clone()
    (_normal(7, 30) @ w).square().sum().backward()
    opt.step()
    assert w.isfinite().all() and not torch.equal(w.detach(), before)

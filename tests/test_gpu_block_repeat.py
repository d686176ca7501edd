"""The gated block and orthogonalised matrices give the same bits every time, whatever ran in between and whatever their outputs and workspaces
held before."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _normal(*shape, dtype=torch.float32, seed=0, unit=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=gen, device=DEV) * unit).to(dtype)


def _spoil():
    """Leaves other numbers, NaN among them, in the memory that the next call is given."""
    for n in (1 << 12, 1 << 20, 1 << 24, 3 << 25):
        torch.full((n,), float("nan"), device=DEV)


@pytest.mark.parametrize("fine", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t,d,h,o", [(4201, 264, 1030, 300), (70, 33, 500, 41), (9, 300, 700, 90)])
def test_gated(t, d, h, o, dtype, fine):
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu = _normal(t, d, dtype=dtype), _normal(h, d, dtype=dtype, seed=1, unit=d ** -0.5), _normal(h, d, dtype=dtype, seed=2, unit=d ** -0.5)
    wd, gy = _normal(o, h, dtype=dtype, seed=3, unit=h ** -0.5), _normal(t, o, dtype=dtype, seed=4)

    def run():
        _spoil()
        y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True, fine=fine)
        _spoil()
        return [y, fsa.fsa_gated_fwd(x, wg, wu, wd, fine=fine), *fsa.fsa_gated_bwd(gy, x, wg, wu, wd, kept, fine=fine),
                *fsa.fsa_gated_bwd(gy, x, wg, wu, wd, fine=fine)]

    first = run()
    assert all(v.isfinite().all() for v in first)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


@pytest.mark.parametrize("b,m,n", [(1, 65, 63), (3, 300, 1400), (1, 1030, 1100), (9, 700, 300)])
def test_orthogonal(b, m, n):
    from paper_2511_13645_amd import binding as fsa
    g = _normal(b, m, n)
    first = fsa.fsa_orthogonalize(g)
    for _ in range(3):
        _spoil()
        assert torch.equal(fsa.fsa_orthogonalize(g), first)

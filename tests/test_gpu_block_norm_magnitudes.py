"""The residual norm of rows whose squares fp32 cannot hold: with no eps a row's magnitude changes nothing, and with one the row is what it
is in 64 bits."""
import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WIDTHS = [1, 7, 60, 300, 1024, 3000, 16384]


def _inputs(t, d, dtype):
    gen = torch.Generator(device=DEV).manual_seed(d)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    # elements of [1, 2), whose power of two is exact
    x = (1.0 + torch.rand((t, d), generator=gen, device=DEV)) * n(t, d).sign()
    return x.to(dtype), (1 + 0.2 * n(d)).to(dtype), n(t, d).to(dtype)


def _times(x, power):
    return (x.double() * 2.0 ** power).to(x.dtype)


@pytest.mark.parametrize("power", [-120, -90, -60, 60, 70, 100, 120])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_power_of_two_changes_nothing(dtype, d, power):
    from paper_2511_13645_amd import binding as fsa
    x, w, gy = _inputs(9, d, dtype)
    y, _ = fsa.fsa_norm_fwd(x, w, None, 0.0)
    bb.check("y", y, *bb.norm(x, None, w, gy, None, 0.0, dtype)["y"])
    gx, gw = fsa.fsa_norm_bwd(gy, None, x, w, 0.0)
    # one row as it is among those that are not: the same wave has both
    big = _times(x, power)
    big[4] = x[4]
    z, _ = fsa.fsa_norm_fwd(big, w, None, 0.0)
    assert torch.equal(z, y)
    hx, hw = fsa.fsa_norm_bwd(gy, None, big, w, 0.0)
    assert torch.equal(hw, gw)
    want = _times(gx, -power)
    want[4] = gx[4]
    # (2^-100 of a small gradient may be subnormal, and is rounded once more: bfloat16's smallest number is 2^-133)
    assert (hx.double() - want.double()).abs().max().item() <= 2.0 ** -133 if power >= 100 else torch.equal(hx, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [60, 3000])
def test_with_a_residual_and_an_eps(dtype, d):
    from paper_2511_13645_amd import binding as fsa
    x, w, gy = _inputs(6, d, dtype)
    r = _inputs(6, d, dtype)[2]
    for unit, eps in ((2.0 ** 100, 1e-6), (2.0 ** -90, 2.0 ** -100), (2.0 ** -90, 1e-6), (2.0 ** 70, 1e30), (2.0 ** -120, 2.0 ** -80), (2.0 ** -75, 2.0 ** -148)):
        a, b = (_times(v, torch.tensor(unit).log2().item()) for v in (x, r))
        want = bb.norm(a, b, w, gy, None, eps, dtype)
        y, s = fsa.fsa_norm_fwd(a, w, b, eps)
        bb.check("s", s, *want["s"])
        bb.check("y", y, *want["y"])
        gx, gw = fsa.fsa_norm_bwd(gy, None, s, w, eps)
        bb.check("grad_weight", gw, *want["grad_weight"])
        bb.check("grad_x", gx, *want["grad_x"])


@pytest.mark.parametrize("d", [40, 500, 5000])
def test_rows_that_are_not_finite_stay_by_themselves(d):
    from paper_2511_13645_amd import binding as fsa
    x, w, gy = _inputs(12, d, torch.float32)
    big = _times(x, 100)
    y0, _ = fsa.fsa_norm_fwd(big, w, None, 0.0)
    big[3, 1], big[7, 2] = float("inf"), float("nan")
    y, _ = fsa.fsa_norm_fwd(big, w, None, 0.0)
    keep = torch.ones(12, dtype=torch.bool, device=DEV)
    keep[3] = keep[7] = False
    assert torch.equal(y[keep], y0[keep]) and y[7].isnan().all() and y[3, 1].isnan()
    zero = torch.zeros_like(x)
    assert torch.equal(fsa.fsa_norm_fwd(zero, w, None, 1e-30)[0], zero)

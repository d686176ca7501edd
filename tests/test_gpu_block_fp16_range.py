"""The gated block in fp16 where what lies between its products is beyond fp16's range, above or below, and the results are not: against the
definition in 64 bits within the bounds of block_bounds.py."""
import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16 = torch.float16
ROWS = [1, 16, 17, 300]


def _inputs(t, d, h, o, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    return [n(t, d), n(h, d) * d ** -0.5, n(h, d) * d ** -0.5, n(o, h) * h ** -0.5, n(t, o)]


def _check(x, wg, wu, wd, gy, act="silu", exact_rows=None):
    from paper_2511_13645_amd import binding as fsa
    want = bb.gated(x, wg, wu, wd, gy, act, F16)
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act, emit_kept=True)
    bb.check("y beside what is kept", y, *want["y"])
    bb.check("y", fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act), *want["y"])
    for given in (None, kept):
        for name, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given, activation=act)):
            bb.check(name, g, *want[name])
    return want


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("t", ROWS)
def test_act_times_u_beyond_fp16(t, act):
    x, wg, wu, wd, gy = _inputs(t, 48, 80, 33)
    x, wg, wu, wd, gy = (v.to(F16) for v in (x, wg * 2000, wu * 2000, wd * 2.0 ** -14, gy * 2.0 ** -6))
    g, u = x.double() @ wg.double().T, x.double() @ wu.double().T
    assert (bb.activation(act, g)[0] * u).abs().max().item() > 65504
    want = _check(x, wg, wu, wd, gy, act)
    # (the gradient of w_down is a sum of such products, and beyond fp16 itself)
    assert all(v.abs().max().item() < 60000 for name, (v, _) in want.items() if name != "grad_down")


@pytest.mark.parametrize("t", ROWS)
def test_act_times_u_below_fp16(t):
    """2^-24 is fp16's smallest number; results are off by little more than their own rounding all the same."""
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(t, 48, 80, 33, seed=1)
    x, wg, wu, wd, gy = (v.to(F16) for v in (x, wg * 2.0 ** -12, wu * 2.0 ** -10, wd * 2.0 ** 13, gy))
    want = bb.gated(x, wg, wu, wd, gy, "silu", F16)
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True)
    down = [fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given)[3] for given in (None, kept)]
    for got, value in [(y, want["y"][0]), (fsa.fsa_gated_fwd(x, wg, wu, wd), want["y"][0])]:
        assert (got.double() - value).norm().item() <= bb.HALF_STEP[F16] * value.norm().item()
    for got in down:                                         # (which itself lies among fp16's subnormal numbers)
        value = want["grad_down"][0]
        assert ((got.double() - value).abs() <= bb.rounding(value, F16) + 2.0 ** -12 * value.abs().max()).all()


@pytest.mark.parametrize("unit", [2.0 ** -16, 2.0 ** -8, 1.0])
@pytest.mark.parametrize("t", ROWS)
def test_gradients_on_the_way_beyond_fp16(t, unit):
    """dh u act' is 2^16 and more times the largest gradient, whatever scale that has; x brings the tables' gradients back."""
    x, wg, wu, wd, gy = _inputs(t, 64, 96, 512, seed=2)
    x, wg, wu, wd, gy = (v.to(F16) for v in (x * 2.0 ** -8, wg * 2.0 ** 8, wu * 2.0 ** 15, wd * 300, gy * unit))
    dh = gy.double() @ wd.double()
    u = x.double() @ wu.double().T
    assert (dh * u).abs().max().item() > 2.0 ** 16 * gy.double().abs().max().item()
    _check(x, wg, wu, wd, gy)


def test_one_large_gradient_leaves_the_others():
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(200, 64, 96, 48, seed=3)
    gy[77] = gy[77].sign() * 60000.0
    x, wg, wu, wd, gy = (v.to(F16) for v in (x, wg, wu, wd, gy))
    want = bb.gated(x, wg, wu, wd, gy, "silu", F16)["grad_x"][0]
    _, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True)
    others = torch.arange(200, device=DEV) != 77
    for given in (None, kept):
        gx = fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given)[0].double()
        # a rounding of half a step of the result and what two numbers leave of dg and du
        assert ((gx - want)[others].norm(dim=1) <= bb.HALF_STEP[F16] * want[others].norm(dim=1)).all()


def test_sizes_of_every_length():
    """Rows of one element and of many, columns that end inside a workgroup's, strides: the search for the longest rows reads what is there
    and nothing else."""
    from paper_2511_13645_amd import binding as fsa
    for t, d, h, o in ((40, 1, 1, 1), (70, 7, 65, 130), (20, 1030, 66, 9), (5000, 3, 129, 2), (33, 520, 63, 257)):
        tensors = [v.to(F16) for v in _inputs(t, d, h, o, seed=t)]
        want = bb.gated(*tensors, "silu", F16)
        wide = [torch.full((v.shape[0] + 2, v.shape[1] + 11), float("inf"), dtype=F16, device=DEV)[1:-1, 3:3 + v.shape[1]] for v in tensors]
        for v, w in zip(tensors, wide):
            w.copy_(v)
        for x, wg, wu, wd, gy in (tensors, wide):
            bb.check("y", fsa.fsa_gated_fwd(x, wg, wu, wd), *want["y"])
            for name, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), fsa.fsa_gated_bwd(gy, x, wg, wu, wd)):
                bb.check(name, g, *want[name])


def test_rows_that_are_not_finite_do_not_count():
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = (v.to(F16) for v in _inputs(90, 40, 56, 24, seed=5))
    y0, g0 = fsa.fsa_gated_fwd(x, wg, wu, wd), fsa.fsa_gated_bwd(gy, x, wg, wu, wd)
    x[3, 0] = float("inf")
    x[50] = float("nan")
    gy[70, 1] = float("-inf")
    keep = torch.ones(90, dtype=torch.bool, device=DEV)
    keep[3] = keep[50] = False
    y = fsa.fsa_gated_fwd(x, wg, wu, wd)
    assert torch.equal(y[keep], y0[keep]) and not y[~keep].isfinite().any()
    keep[70] = False
    gx = fsa.fsa_gated_bwd(gy, x, wg, wu, wd)[0]
    assert torch.equal(gx[keep], g0[0][keep]) and not gx[~keep].isfinite().any()
    w = wg.clone()
    w[7, 3] = float("inf")                                   # a gate that is not finite in any row
    assert not fsa.fsa_gated_fwd(x, w, wu, wd).isfinite().any()


def test_zeros():
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = (v.to(F16) for v in _inputs(50, 40, 56, 24))
    for zero in range(5):
        tensors = [x, wg, wu, wd, gy]
        tensors[zero] = torch.zeros_like(tensors[zero])
        want = bb.gated(*tensors, "silu", F16)
        bb.check("y", fsa.fsa_gated_fwd(*tensors[:4]), *want["y"])
        for name, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), fsa.fsa_gated_bwd(tensors[4], *tensors[:4])):
            bb.check(name, g, *want[name])

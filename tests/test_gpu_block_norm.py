"""The residual norm against its definition in 64 bits: every type, odd widths, strides, one row and none, gradients given and
not, other streams, a captured graph; what it refuses is in test_block_refusals.py."""
import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(t, d, dtype, seed=0, wdtype=None):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    return (n(t, d).to(dtype), (n(t, d) * 2).to(dtype), (1 + 0.2 * n(d)).to(wdtype or dtype), n(t, d).to(dtype), n(t, d).to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,d", [(1, 1), (3, 2), (2, 7), (65, 16), (17, 64), (33, 65), (1024, 128), (5, 256), (130, 257), (77, 602),
                                 (9, 1024), (4, 1025), (300, 2048), (3, 4096), (2, 4097), (5, 16384), (1, 16383)])
def test_rows_and_gradients(t, d, dtype):
    from paper_2511_13645_amd.autograd import fused_residual_norm
    x, r, w, gy, gs = _inputs(t, d, dtype, seed=t + d)
    for u in (x, r, w):
        u.requires_grad_(True)
    want = bb.norm(x, r, w, gy, gs, 1e-6, dtype)
    y, s = fused_residual_norm(x, w, r, eps=1e-6)
    assert torch.equal(s.detach().double(), want["s"][0])
    bb.check("y", y, *want["y"])
    gx, gr, gw = torch.autograd.grad((y, s), (x, r, w), (gy, gs))
    assert torch.equal(gx, gr)
    bb.check("grad_x", gx, *want["grad_x"])
    bb.check("grad_weight", gw, *want["grad_weight"])
    # without a residual, and with the gradient of one output alone
    alone = bb.norm(x, None, w, gy, None, 1e-6, dtype)
    y, s = fused_residual_norm(x, w, eps=1e-6)
    assert s is x
    bb.check("y alone", y, *alone["y"])
    gx, gw = torch.autograd.grad(y, (x, w), gy)
    bb.check("grad_x alone", gx, *alone["grad_x"])
    bb.check("grad_weight alone", gw, *alone["grad_weight"])
    y, s = fused_residual_norm(x, w, r, eps=1e-6)
    gx, = torch.autograd.grad(s, (x,), gs)
    assert torch.equal(gx, gs)


@pytest.mark.parametrize("dtype,wdtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.float16), (torch.float16, torch.bfloat16)])
def test_weight_of_another_type(dtype, wdtype):
    from paper_2511_13645_amd import binding as fsa
    x, r, w, gy, gs = _inputs(50, 300, dtype, wdtype=wdtype)
    want = bb.norm(x, r, w, gy, gs, 1e-5, dtype)
    y, s = fsa.fsa_norm_fwd(x, w, r, 1e-5)
    gx, gw = fsa.fsa_norm_bwd(gy, gs, s, w, 1e-5)
    assert gw.dtype == wdtype
    for name, got in (("y", y), ("grad_x", gx), ("grad_weight", gw)):
        bb.check(name, got, *want[name])
    assert fsa.fsa_norm_bwd(gy, gs, s, w, 1e-5, want_x=False)[0] is None
    assert fsa.fsa_norm_bwd(gy, gs, s, w, 1e-5, want_weight=False)[1] is None


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows_off_the_grid_leave_their_surroundings(dtype):
    from paper_2511_13645_amd import binding as fsa
    t, d = 37, 99
    x, r, w, gy, gs = _inputs(t, d, dtype)
    wide = torch.full((t, 3 * d + 5), 7.0, dtype=dtype, device=DEV)
    xs, rs = wide[:, 3:3 + d], wide[:, d + 4:2 * d + 4]
    xs.copy_(x)
    rs.copy_(r)
    before = wide.clone()
    y, s = fsa.fsa_norm_fwd(xs, w, rs, 1e-6)
    y0, s0 = fsa.fsa_norm_fwd(x, w, r, 1e-6)
    assert torch.equal(y, y0) and torch.equal(s, s0) and torch.equal(wide, before)
    a, b = fsa.fsa_norm_bwd(gy, gs, xs, w), fsa.fsa_norm_bwd(gy, gs, x, w)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_rows_and_rows_of_zeros():
    from paper_2511_13645_amd import binding as fsa
    w = torch.ones(40, device=DEV)
    e = torch.empty((0, 40), device=DEV)
    y, s = fsa.fsa_norm_fwd(e, w, e)
    assert y.shape == (0, 40) and s.shape == (0, 40)
    gx, gw = fsa.fsa_norm_bwd(e, e, e, w)
    assert gx.shape == (0, 40) and torch.equal(gw, torch.zeros_like(w))
    z = torch.zeros((5, 40), device=DEV)
    y, _ = fsa.fsa_norm_fwd(z, w)
    assert torch.equal(y, z)
    gx, gw = fsa.fsa_norm_bwd(torch.ones_like(z), None, z, w, 1e-6)
    assert torch.allclose(gx, torch.full_like(z, 1e3)) and torch.equal(gw, torch.zeros_like(w))


def test_a_row_that_is_not_finite_stays_by_itself():
    from paper_2511_13645_amd import binding as fsa
    x, r, w, gy, gs = _inputs(20, 200, torch.float32)
    y0, s0 = fsa.fsa_norm_fwd(x, w, r)
    x[7, 3] = float("nan")
    x[11, 5] = float("inf")
    y, s = fsa.fsa_norm_fwd(x, w, r)
    keep = torch.ones(20, dtype=torch.bool, device=DEV)
    keep[7] = keep[11] = False
    assert torch.equal(y[keep], y0[keep]) and torch.equal(s[keep], s0[keep])
    assert y[7].isnan().all() and y[11, 5].isnan()


def test_gradients_agree_with_differences():
    from paper_2511_13645_amd.autograd import fused_residual_norm
    x, r, w, gy, gs = _inputs(3, 24, torch.float32, seed=5)
    for u in (x, r, w):
        u.requires_grad_(True)
    value = lambda: sum((a.double() * b.double()).sum() for a, b in zip(fused_residual_norm(x, w, r, eps=1e-3), (gy, gs)))
    grads = torch.autograd.grad(value(), (x, r, w))
    step = 2.0 ** -8                                        # error: step^2 / 6 of the third derivative, and 2^-24 / step of the values
    for t, g in zip((x, r, w), grads):
        for i in range(0, t.numel(), 11):
            with torch.no_grad():
                at = t.view(-1)[i].item()
                t.view(-1)[i] = at + step
                up = value().item()
                t.view(-1)[i] = at - step
                down = value().item()
                t.view(-1)[i] = at
            assert abs((up - down) / (2 * step) - g.reshape(-1)[i].item()) < 2e-3


def test_results_do_not_change_from_call_to_call():
    from paper_2511_13645_amd import binding as fsa
    x, r, w, gy, gs = _inputs(5000, 130, torch.bfloat16)
    y, s = fsa.fsa_norm_fwd(x, w, r)
    first = fsa.fsa_norm_bwd(gy, gs, s, w)
    for _ in range(3):
        again = fsa.fsa_norm_bwd(gy, gs, s, w)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])

"""The gated feed-forward block against its definition in 64 bits, element by element within the bounds of block_bounds.py: every
type and activation, sizes around the tiles' edges, strides, no rows, gradients that are not wanted, not finite rows, differences."""
import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(t, d, h, o, dtype, seed=0, unit=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    return (n(t, d).to(dtype), (n(h, d) * 1.5 * d ** -0.5).to(dtype), (n(h, d) * 1.5 * d ** -0.5).to(dtype),
            (n(o, h) * h ** -0.5).to(dtype), (n(t, o) * unit).to(dtype))


def _check(x, wg, wu, wd, gy, act, dtype):
    from paper_2511_13645_amd import binding as fsa
    want = bb.gated(x, wg, wu, wd, gy, act, dtype)
    y = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act)
    bb.check("y", y, *want["y"])
    again, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act, emit_kept=True)
    bb.check("y beside what is kept", again, *want["y"])
    for given in (None, kept):
        got = fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given, activation=act)
        for name, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), got):
            bb.check(name, g, *want[name])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,d,h,o", [(1, 1, 1, 1), (1, 64, 64, 64), (2, 3, 5, 7), (16, 16, 32, 16), (17, 100, 333, 47), (33, 8, 1000, 9),
                                     (63, 65, 66, 67), (64, 64, 64, 64), (65, 128, 129, 127), (127, 602, 130, 31), (128, 256, 512, 256),
                                     (129, 24, 40, 264), (300, 136, 520, 72), (1000, 33, 70, 33), (5, 1024, 2048, 1024)])
def test_sizes(t, d, h, o, dtype):
    _check(*_inputs(t, d, h, o, dtype, seed=t + h), "silu", dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["gelu", "relu"])
@pytest.mark.parametrize("t,d,h,o", [(1, 40, 50, 60), (70, 90, 110, 130), (513, 64, 200, 47)])
def test_activations(t, d, h, o, act, dtype):
    _check(*_inputs(t, d, h, o, dtype, seed=h), act, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_tiles_of_every_width_and_split_depths(dtype):
    # as many tiles as take the wide ones; a depth (rows) that the weights' gradients split
    _check(*_inputs(4200, 72, 1030, 40, dtype), "silu", dtype)
    _check(*_inputs(9001, 40, 56, 24, dtype, unit=1e-3), "silu", dtype)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", TYPES)
def test_gates_far_from_zero(act, dtype):
    x, wg, wu, wd, gy = _inputs(64, 32, 96, 48, dtype, seed=3)
    _check((x.float() * 8).to(dtype), (wg.float() * 4).to(dtype), (wu.float() / 8).to(dtype), wd, gy, act, dtype)


@pytest.mark.parametrize("unit", [2.0 ** -20, 2.0 ** -14, 1.0, 2.0 ** 12])
def test_fp16_gradients_of_any_scale(unit):
    _check(*_inputs(90, 48, 100, 30, torch.float16, seed=9, unit=unit), "silu", torch.float16)


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_operands_off_the_grid(dtype):
    from paper_2511_13645_amd import binding as fsa
    t, d, h, o = 70, 50, 90, 41
    tensors = _inputs(t, d, h, o, dtype, seed=2)
    room = [torch.full((m.shape[0], m.shape[1] * 2 + 9), 3.0, dtype=dtype, device=DEV) for m in tensors]
    views = [r[:, 5:5 + m.shape[1]] for r, m in zip(room, tensors)]
    for v, m in zip(views, tensors):
        v.copy_(m)
    before = [r.clone() for r in room]
    assert torch.equal(fsa.fsa_gated_fwd(*views[:4]), fsa.fsa_gated_fwd(*tensors[:4]))
    a, b = fsa.fsa_gated_bwd(views[4], *views[:4]), fsa.fsa_gated_bwd(tensors[4], *tensors[:4])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert all(torch.equal(p, q) for p, q in zip(room, before))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_on_the_grid_with_room_between_them(dtype):
    from paper_2511_13645_amd import binding as fsa
    tensors = _inputs(200, 64, 128, 72, dtype, seed=4)
    views = [torch.full((m.shape[0], m.shape[1] + 24), float("nan"), dtype=dtype, device=DEV)[:, 8:8 + m.shape[1]] for m in tensors]
    for v, m in zip(views, tensors):
        v.copy_(m)
    assert torch.equal(fsa.fsa_gated_fwd(*views[:4]), fsa.fsa_gated_fwd(*tensors[:4]))
    a, b = fsa.fsa_gated_bwd(views[4], *views[:4]), fsa.fsa_gated_bwd(tensors[4], *tensors[:4])
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(0, 24, 40, 16, dtype)
    assert fsa.fsa_gated_fwd(x, wg, wu, wd).shape == (0, 16)
    gx, *rest = fsa.fsa_gated_bwd(gy, x, wg, wu, wd)
    assert gx.shape == (0, 24)
    assert all(torch.equal(g, torch.zeros_like(w)) for g, w in zip(rest, (wg, wu, wd)))


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_that_are_not_wanted(dtype):
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(150, 40, 88, 56, dtype)
    whole = fsa.fsa_gated_bwd(gy, x, wg, wu, wd)
    for mask in range(16):
        want = [bool(mask >> i & 1) for i in range(4)]
        some = fsa.fsa_gated_bwd(gy, x, wg, wu, wd, want=want)
        for w, a, b in zip(want, some, whole):
            assert a is None if not w else torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_that_is_not_finite_stays_by_itself(dtype):
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(100, 44, 70, 36, dtype)
    y0, gx0 = fsa.fsa_gated_fwd(x, wg, wu, wd), fsa.fsa_gated_bwd(gy, x, wg, wu, wd)[0]
    x[13, 43] = float("nan")
    x[77, 0] = float("inf")
    gy[50, 35] = float("nan")
    keep = torch.ones(100, dtype=torch.bool, device=DEV)
    keep[13] = keep[77] = False
    y = fsa.fsa_gated_fwd(x, wg, wu, wd)
    assert torch.equal(y[keep], y0[keep]) and y[13].isnan().all()
    keep[50] = False
    gx = fsa.fsa_gated_bwd(gy, x, wg, wu, wd)[0]
    assert torch.equal(gx[keep], gx0[keep]) and gx[13].isnan().all() and gx[50].isnan().all()


def test_fp32_elements_of_every_magnitude():
    # rows and columns hundreds of binades apart: planes keep 24 bits wherever an element lies
    x, wg, wu, wd, gy = _inputs(40, 32, 64, 24, torch.float32, seed=8)
    x = x * torch.logspace(-9, 3, 40, device=DEV)[:, None]
    wg = wg * torch.logspace(-3, 0, 32, device=DEV)[None, :]
    wd = wd * torch.logspace(-12, 6, 24, device=DEV)[:, None]
    gy = gy * torch.logspace(-15, 0, 40, device=DEV)[:, None]
    _check(x, wg, wu, wd, gy, "silu", torch.float32)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gradients_agree_with_differences(act):
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward
    tensors = [t.requires_grad_(True) for t in _inputs(3, 12, 20, 8, torch.float32, seed=1)[:4]]
    gy = _inputs(3, 12, 20, 8, torch.float32, seed=1)[4]
    value = lambda: (fused_gated_feed_forward(*tensors, activation=act).double() * gy.double()).sum()
    grads = torch.autograd.grad(value(), tensors)
    step = 2.0 ** -7
    for t, g in zip(tensors, grads):
        for i in range(0, t.numel(), 13):
            with torch.no_grad():
                at = t.view(-1)[i].item()
                if act == "relu":                            # only where no gate changes its sign on the way
                    t.view(-1)[i] = at - step
                    low = tensors[0] @ tensors[1].T > 0
                    t.view(-1)[i] = at + step
                    if not torch.equal(low, tensors[0] @ tensors[1].T > 0):
                        t.view(-1)[i] = at
                        continue
                t.view(-1)[i] = at + step
                up = value().item()
                t.view(-1)[i] = at - step
                down = value().item()
                t.view(-1)[i] = at
            # step^2 / 6 = 1e-5 of third derivatives of a few units, and 2^-22 / step = 3e-5 of the values' rounding
            assert abs((up - down) / (2 * step) - g.reshape(-1)[i].item()) < 2e-3


def test_gradients_through_autograd_in_every_form():
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward
    x, wg, wu, wd, gy = _inputs(60, 24, 48, 24, torch.float32)
    leaves = [t.requires_grad_(True) for t in (x, wg, wu, wd)]
    y = fused_gated_feed_forward(*leaves)
    whole = torch.autograd.grad(y, leaves, torch.ones_like(y))
    again = torch.autograd.grad(fused_gated_feed_forward(*leaves).sum(), leaves)        # a gradient that is a broadcast one
    assert all(torch.equal(a, b) for a, b in zip(whole, again))
    # one matrix in both places: the gradient is the sum
    both = torch.autograd.grad(fused_gated_feed_forward(x, wg, wg, wd), (wg,), torch.ones_like(y))[0]
    apart = torch.autograd.grad(fused_gated_feed_forward(x, wg, wg.detach().clone().requires_grad_(True), wd), (wg,), torch.ones_like(y))[0]
    other = wg.detach().clone().requires_grad_(True)
    up = torch.autograd.grad(fused_gated_feed_forward(x, wg.detach(), other, wd), (other,), torch.ones_like(y))[0]
    assert torch.allclose(both, apart + up, rtol=0, atol=2e-7 * both.abs().max().item() * 4)
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(fused_gated_feed_forward(*leaves).sum(), (x,), create_graph=True)
        g.sum().backward()

"""What the gated block holds between its products, as the caller chooses it: with `fine`, and wherever a call has few rows, 16-bit
results are off by their own rounding alone, in large calls too, whether a gradient is wanted or not."""
import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# rows, D, H, O: of 4e9 operations and more, where one number of the type lies between the products unless the call is fine
LARGE = [(4000, 264, 520, 264), (2100, 100, 1500, 90), (1030, 400, 1100, 520)]


def _inputs(t, d, h, o, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    return (n(t, d).to(dtype), (n(h, d) * 1.5 * d ** -0.5).to(dtype), (n(h, d) * 1.5 * d ** -0.5).to(dtype),
            (n(o, h) * h ** -0.5).to(dtype), n(t, o).to(dtype))


def _exact(x, wg, wu, wd, gy):
    leaves = [t.double().requires_grad_(True) for t in (x, wg, wu, wd)]
    y = (torch.nn.functional.silu(leaves[0] @ leaves[1].T) * (leaves[0] @ leaves[2].T)) @ leaves[3].T
    return [y.detach(), *torch.autograd.grad(y, leaves, gy.double())]


def _off(got, want):
    return [((g.detach().double() - w).norm() / w.norm()).item() for g, w in zip(got, want)]


def _own(dtype):
    # A rounding is uniform within half a step, which relative to the numbers' mean square is 1 / sqrt(3) of that of the type by the
    # mean square of (binade's foot / number): 0.65 to 0.74 for numbers spread evenly over a binade, evenly by their logarithm, or
    # normal.  What two numbers of the type leave is 2^-8 of that, and fp32 sums less: within 1.1 in all, where one of a factor as well
    # makes sqrt(2) of it.
    return bb.HALF_STEP[dtype] / 3 ** 0.5 * 0.74 * 1.1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t,d,h,o", LARGE)
def test_fine_results_have_their_own_rounding_alone(t, d, h, o, dtype):
    from paper_2511_13645_amd import binding as fsa
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward
    assert 6 * t * h * (2 * d + o) >= 4e9
    x, wg, wu, wd, gy = _inputs(t, d, h, o, dtype)
    want = _exact(x, wg, wu, wd, gy)
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True, fine=True)
    assert kept.numel() > fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True)[1].numel()
    assert torch.equal(y, fsa.fsa_gated_fwd(x, wg, wu, wd, fine=True))
    for given in (None, kept):
        assert max(_off([y, *fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given, fine=True)], want)) <= _own(dtype)
    leaves = [v.requires_grad_(True) for v in (x, wg, wu, wd)]
    y = fused_gated_feed_forward(*leaves, fine=True)
    assert max(_off([y, *torch.autograd.grad(y, leaves, gy)], want)) <= _own(dtype)
    y = fused_gated_feed_forward(*leaves)                    # and otherwise one factor's rounding more
    assert max(_off([y, *torch.autograd.grad(y, leaves, gy)], want)) <= 2 ** 0.5 * _own(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_both_host_paths_take_it(dtype, monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward
    x, wg, wu, wd, gy = _inputs(*LARGE[2], dtype)
    leaves = [v.requires_grad_(True) for v in (x, wg, wu, wd)]

    def run():
        y = fused_gated_feed_forward(*leaves, fine=True)
        return [y, *torch.autograd.grad(y, leaves, gy)]

    native = run()
    assert fsa._block_host.gated(*leaves, 0, True) is not None and fsa._block_host.gated_fwd(*leaves, 0, True) is not None
    monkeypatch.setattr(fsa, "_block_host", None)
    assert all(torch.equal(a, b) for a, b in zip(native, run()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t", [1, 9, 16])
def test_few_rows_are_as_exact_whether_a_gradient_is_wanted_or_not(t, dtype):
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(t, 2048, 16384, 2048, dtype)
    assert t < 7 or 6 * t * 16384 * 3 * 2048 >= 4e9
    want = _exact(x, wg, wu, wd, gy)
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True)
    # (a row has 2048 numbers, whose roundings' mean square is off by 2 percent)
    for got in (y, fsa.fsa_gated_fwd(x, wg, wu, wd)):
        assert _off([got], want[:1])[0] <= 1.06 * _own(dtype)
    assert max(_off(fsa.fsa_gated_bwd(gy, x, wg, wu, wd, kept), want[1:])) <= 1.06 * _own(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_room_that_the_caller_is_told(dtype):
    from paper_2511_13645_amd import binding as fsa
    t, d, h, o = LARGE[0]
    x, wg, wu, wd, gy = _inputs(t, d, h, o, dtype)
    for need, call in ((fsa.fsa_gated_fwd_workspace_bytes(t, d, h, o, dtype, fine=True), lambda ws: [fsa.fsa_gated_fwd(x, wg, wu, wd, fine=True, workspace=ws)]),
                       (fsa.fsa_gated_bwd_workspace_bytes(t, d, h, o, dtype, fine=True), lambda ws: fsa.fsa_gated_bwd(gy, x, wg, wu, wd, fine=True, workspace=ws))):
        ws = torch.full((need + 512,), 7, dtype=torch.uint8, device=DEV)
        first = call(ws[:need])
        assert (ws[need:] == 7).all() and all(torch.equal(a, b) for a, b in zip(first, call(None)))


def test_what_is_kept_belongs_to_the_choice():
    from paper_2511_13645_amd import binding as fsa
    x, wg, wu, wd, gy = _inputs(*LARGE[0], torch.bfloat16)
    _, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True, fine=True)
    with pytest.raises(ValueError):
        fsa.fsa_gated_bwd(gy, x, wg, wu, wd, kept)

"""Gates far below zero, alone: what an activation leaves of them is small but has as many bits as any other number.

One row, one hidden element: every product is of two numbers, so that act * u is off by what the activation is, and y and the gradients
by a few roundings to the type: of h, dg or du and of themselves.  v = 2^-24: an exponential whose argument is off by 2 v of itself
(g, or g^2 / 2 in the tail of the normal distribution, and a constant) is off by 2 v times that argument, and by the functions' own few v (16 beside 16-bit types).  fp16 has no number between those that lie
2^-24 apart, beside which dg and du are held to 2^-25 of gradients of one."""
import math

import pytest
import torch

import block_bounds as bb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t", [1, 40])
def test_tails(t, act, dtype):
    from paper_2511_13645_amd import binding as fsa
    one = torch.ones((1, 1), dtype=dtype, device=DEV)
    gates = [-0.5, -1.0, -2.0, -3.0, -4.0, -5.0, -5.5, -6.0, -8.0]
    if dtype != torch.float16:
        gates += [-9.5]
    for gate in gates:
        g = torch.tensor([[gate]], dtype=dtype, device=DEV)
        value, slope, _, _ = bb.activation(act, g.double())
        # u brings act * u to about one, or as near as the type has numbers for it
        u = torch.tensor([[2.0 ** min(14, round(-math.log2(value.abs().item())))]], dtype=dtype, device=DEV)
        x = one.expand(t, 1).contiguous()
        y, kept = fsa.fsa_gated_fwd(x, g, u, one, activation=act, emit_kept=True)
        got = [fsa.fsa_gated_fwd(x, g, u, one, activation=act), y]
        h = (value * u.double()).expand(t, 1)
        if h.abs().min().item() < 2.0 ** -13 and dtype == torch.float16:
            continue
        function = ((8 if dtype == torch.float32 else 16) + 2 * max(abs(gate), gate * gate)) * bb.V
        bound = 3 * bb.HALF_STEP[dtype] + function
        for a in got:
            assert ((a.double() - h).abs() <= bound * h.abs()).all(), (gate, a[0].item(), h[0].item())
        for given in (None, kept):
            gx, gg, gu, gd = fsa.fsa_gated_bwd(x, x, g, u, one, given, activation=act)
            want = ((u.double() * slope), (value.double()), h[:1])
            # p + g bell and p (1 + g (1 - p)) are sums of either sign that lose up to 3 bits where the slope is near zero (-0.75, -1.28)
            steps = 8 if abs((slope / value).item()) < 2 else 1
            for name, a, w in (("grad_gate", gg, want[0] * t), ("grad_up", gu, want[1] * t), ("grad_down", gd, want[2] * t)):
                assert (a.double() - w).abs().max().item() <= (bound + steps * function) * w.abs().max().item() + (t + 1) * bb.FLOOR[dtype], (name, gate)

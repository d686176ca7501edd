"""Every tile of the gated block and of orthogonalised matrices (block_tiles.py) against the definitions in 64 bits, and orthogonalised
matrices direction by direction."""
import pytest
import torch

import block_bounds as bb
import block_tiles as tiles
import test_gpu_block_orthogonal as ortho

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CASES = [(kind, *case) for kind, cases in tiles.GATED.items() for case in cases] + [(kind, *case) for kind in ("bf16", "f16") for case in tiles.IN_PLACE]


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("kind,fine,t,d,h,o", CASES)
def test_gated(kind, fine, t, d, h, o, act):
    from paper_2511_13645_amd import binding as fsa
    dtype = TYPES[kind]
    gen = torch.Generator(device=DEV).manual_seed(t + d + h + o)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    x, wg, wu, wd, gy = (v.to(dtype) for v in (n(t, d), n(h, d) * 1.5 * d ** -0.5, n(h, d) * 1.5 * d ** -0.5, n(o, h) * h ** -0.5, n(t, o)))
    want = bb.gated(x, wg, wu, wd, gy, act, dtype)
    bb.check("y", fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act, fine=fine), *want["y"])
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, activation=act, fine=fine, emit_kept=True)
    bb.check("y beside what is kept", y, *want["y"])
    for given in (None, kept):
        for name, g in zip(("grad_x", "grad_gate", "grad_up", "grad_down"), fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given, activation=act, fine=fine)):
            bb.check(name, g, *want[name])


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("b,m,n", tiles.ORTHOGONAL)
def test_orthogonal(b, m, n, kind):
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(m + n)
    g = torch.randn((b, m, n), generator=gen, device=DEV).to(TYPES[kind])
    ortho._check(fsa.fsa_orthogonalize(g, ortho.ABC, 2), ortho._reference(g, [ortho.ABC] * 2), 2, g.dtype)


@pytest.mark.parametrize("b,m,n", [(1, 65, 130), (29, 131, 129), (57, 259, 257), (18, 193, 1291)])
def test_weak_directions_beside_strong_ones(b, m, n):
    """Singular values from one down to a ten thousandth: along each pair of directions lies what the polynomials make of its own, off by
    what a step's products are off by in any one direction, a number of 2^-24 of what they add up, and nothing of the others."""
    from paper_2511_13645_amd import binding as fsa
    gen = torch.Generator(device=DEV).manual_seed(m)
    r = min(m, n)
    u, _ = torch.linalg.qr(torch.randn((b, m, r), generator=gen, device=DEV, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn((b, n, r), generator=gen, device=DEV, dtype=torch.float64))
    sigma = torch.logspace(0, -4, r, device=DEV, dtype=torch.float64)
    g = torch.bmm(u * sigma, v.mT.contiguous()).float()
    # (of the fp32 matrix, whose rounding is no error of the call's)
    want = ortho._reference(g, [ortho.ABC] * 3, 0.0)
    got = fsa.fsa_orthogonalize(g, ortho.ABC, 3, eps=0.0).double()
    along = lambda a: torch.bmm(torch.bmm(u.mT.contiguous(), a), v)
    off = (along(got) - along(want)).abs()
    # a step rounds X, A and P, 2^-24 of each of their elements at random, and sums up to n products in fp32: along one direction that is
    # 2^-24 of the mean element, some |X|_F / sqrt(r) of the strongest, by the sqrt of the sums' length at most; three steps, slopes up to 3.5
    each = bb.V * sum(map(abs, ortho.ABC)) * (8 + max(m, n) ** 0.5) * want.norm(dim=(-2, -1)).max().item() / r ** 0.5
    assert off.max().item() <= each * (1 + 3.5 + 3.5 ** 2)
    # of which the weakest direction is many times as much
    weakest = along(want).diagonal(dim1=-2, dim2=-1).abs().min().item()
    assert off.max().item() <= 0.05 * weakest

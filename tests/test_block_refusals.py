"""What the block's C entry points refuse, and with which status: validation comes before the first launch, so that no GPU is
needed.  And the Python entry points' own refusals of tensors that do not live on a GPU."""
import ctypes

import pytest
import torch

FAKE = 0x10000   # non-null, 16-byte aligned; never dereferenced on an error path
NULL, ARG, DTYPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def fsa():
    from paper_2511_13645_amd import binding, build
    if build.is_stale():
        build.build_hip()
    return binding


def _norm(fsa, **kw):
    a = dict(x=FAKE, xs=64, r=FAKE, rs=64, w=FAKE, t=0, wt=0, T=8, D=64, eps=1e-6, y=FAKE, s=FAKE)
    a.update(kw)
    return fsa.lib().fsa_norm_fwd(a["x"], a["xs"], a["r"], a["rs"], a["w"], a["t"], a["wt"], a["T"], a["D"], a["eps"], a["y"], a["s"], None)


def test_norm_forward(fsa):
    assert _norm(fsa, x=None) == NULL and _norm(fsa, w=None) == NULL and _norm(fsa, y=None) == NULL and _norm(fsa, s=None) == NULL
    assert _norm(fsa, t=3) == DTYPE and _norm(fsa, wt=-1) == DTYPE
    for bad in (dict(T=-1), dict(T=(1 << 30) + 1), dict(D=0), dict(D=16385, xs=16385, rs=16385), dict(xs=63), dict(rs=63), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(r=None), dict(xs=(1 << 31) + 1)):
        assert _norm(fsa, **bad) == ARG, bad
    for name in ("x", "r", "y", "s", "w"):
        assert _norm(fsa, **{name: FAKE + 2}) == ALIGN
        assert _norm(fsa, t=1, wt=1, **{name: FAKE + 1}) == ALIGN
    assert _norm(fsa, T=0, x=None, r=None, y=None, s=None) == 0


def _norm_bwd(fsa, **kw):
    a = dict(gy=FAKE, gs=FAKE, s=FAKE, ss=64, w=FAKE, t=0, wt=0, T=8, D=64, eps=1e-6, gx=FAKE, gw=FAKE, ws=FAKE, n=1 << 30)
    a.update(kw)
    return fsa.lib().fsa_norm_bwd(a["gy"], a["gs"], a["s"], a["ss"], a["w"], a["t"], a["wt"], a["T"], a["D"], a["eps"], a["gx"], a["gw"],
                                  a["ws"], a["n"], None)


def test_norm_backward(fsa):
    assert _norm_bwd(fsa, s=None) == NULL and _norm_bwd(fsa, w=None) == NULL
    assert _norm_bwd(fsa, t=7) == DTYPE and _norm_bwd(fsa, D=0) == ARG and _norm_bwd(fsa, ss=10) == ARG and _norm_bwd(fsa, n=-1) == ARG
    need = fsa.fsa_norm_bwd_workspace_bytes(8, 64, torch.float32)
    assert need > 0
    assert _norm_bwd(fsa, n=need - 1) == WORKSPACE and _norm_bwd(fsa, ws=None) == WORKSPACE and _norm_bwd(fsa, ws=FAKE + 4) == ALIGN
    for name in ("gy", "gs", "s", "w", "gx", "gw"):
        assert _norm_bwd(fsa, **{name: FAKE + 2}) == ALIGN
    assert _norm_bwd(fsa, T=0, s=None, gw=None, gx=None, ws=None, n=0) == 0
    assert _norm_bwd(fsa, gw=None, gx=None, ws=None, n=0) == 0
    assert fsa.lib().fsa_norm_bwd_workspace_bytes(8, 64, 9) == 0 and fsa.lib().fsa_norm_bwd_workspace_bytes(8, 0, 0) == 0


def _gated(fsa, **kw):
    a = dict(x=FAKE, xs=64, g=FAKE, gs=64, u=FAKE, us=64, d=FAKE, ds=128, t=1, act=0, T=8, D=64, H=128, O=32, y=FAKE, k=None, ws=FAKE, n=1 << 40)
    a.update(kw)
    return fsa.lib().fsa_gated_fwd(a["x"], a["xs"], a["g"], a["gs"], a["u"], a["us"], a["d"], a["ds"], a["t"], a["act"], a["T"], a["D"],
                                   a["H"], a["O"], a["y"], a["k"], a["ws"], a["n"], None)


def _gated_bwd(fsa, **kw):
    a = dict(gy=FAKE, gys=32, x=FAKE, xs=64, g=FAKE, gs=64, u=FAKE, us=64, d=FAKE, ds=128, t=1, act=0, T=8, D=64, H=128, O=32, k=FAKE,
             gx=FAKE, gg=FAKE, gu=FAKE, gd=FAKE, ws=FAKE, n=1 << 40)
    a.update(kw)
    return fsa.lib().fsa_gated_bwd(a["gy"], a["gys"], a["x"], a["xs"], a["g"], a["gs"], a["u"], a["us"], a["d"], a["ds"], a["t"], a["act"],
                                   a["T"], a["D"], a["H"], a["O"], a["k"], a["gx"], a["gg"], a["gu"], a["gd"], a["ws"], a["n"], None)


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_gated(fsa, which):
    call = _gated if which == "forward" else _gated_bwd
    for name in ("x", "g", "u", "d", "y" if which == "forward" else "gy"):
        assert call(fsa, **{name: None}) == NULL, name
        assert call(fsa, **{name: FAKE + 1}) == ALIGN, name
    assert call(fsa, t=5) == DTYPE and call(fsa, k=FAKE + 4) == ALIGN
    for bad in (dict(act=-1), dict(act=3), dict(T=-1), dict(T=(1 << 26) + 1), dict(D=0), dict(H=0), dict(O=0), dict(D=65537, xs=65537, gs=65537, us=65537),
                dict(H=65537, ds=65537), dict(xs=63), dict(gs=63), dict(us=0), dict(ds=127), dict(xs=1 << 32)):
        assert call(fsa, **bad) == ARG, bad
    need = getattr(fsa, "fsa_gated_%s_workspace_bytes" % ("fwd" if which == "forward" else "bwd"))
    assert need(8, 64, 128, 32, torch.bfloat16) > 0 and need(8, 0, 128, 32, torch.bfloat16) == 0
    assert call(fsa, n=16) == WORKSPACE and call(fsa, ws=None) == WORKSPACE and call(fsa, ws=FAKE + 8) == ALIGN and call(fsa, n=-1) == ARG
    if which == "forward":
        assert call(fsa, T=0, x=None, y=None, ws=None, n=0) == 0
    else:
        assert call(fsa, gys=31) == ARG
        assert call(fsa, T=0, x=None, gy=None, gg=None, gu=None, gd=None, ws=None, n=0) == 0
        for name in ("gx", "gg", "gu", "gd"):
            assert call(fsa, **{name: FAKE + 1}) == ALIGN


def test_room_for_no_rows_and_for_many(fsa):
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for t in (0, 1, 1 << 26):
            assert fsa.fsa_gated_fwd_workspace_bytes(t, 65536, 65536, 65536, dtype) > 0
            assert fsa.fsa_gated_bwd_workspace_bytes(t, 1, 1, 1, dtype) > 0
        assert fsa.fsa_norm_bwd_workspace_bytes(0, 5, dtype) > 0


def _orthogonal(fsa, **kw):
    a = dict(g=FAKE, bs=64 * 32, s=32, t=0, B=2, M=64, N=32, c=(3.0, -4.0, 2.0), steps=1, eps=1e-7, scale=1.0, out=FAKE, ws=FAKE, n=1 << 40)
    a.update(kw)
    host = None if a["c"] is None else (ctypes.c_float * 96)(*a["c"])
    return fsa.lib().fsa_orthogonalize(a["g"], a["bs"], a["s"], a["t"], a["B"], a["M"], a["N"], host, a["steps"], a["eps"], a["scale"],
                                       a["out"], a["ws"], a["n"], None)


def test_orthogonal(fsa):
    assert _orthogonal(fsa, g=None) == NULL and _orthogonal(fsa, out=None) == NULL and _orthogonal(fsa, c=None) == NULL
    assert _orthogonal(fsa, t=4) == DTYPE
    nan, inf = float("nan"), float("inf")
    for bad in (dict(B=-1), dict(B=65536), dict(M=0), dict(N=0), dict(M=65537), dict(N=65537, s=65537), dict(steps=0), dict(steps=33),
                dict(eps=-1.0), dict(eps=nan), dict(scale=inf), dict(s=31), dict(bs=-1), dict(c=(nan, 0, 0)), dict(c=(0, 17, 0)), dict(c=(0, 0, -inf))):
        assert _orthogonal(fsa, **bad) == ARG, bad
    assert _orthogonal(fsa, g=FAKE + 2) == ALIGN and _orthogonal(fsa, out=FAKE + 1, t=1) == ALIGN and _orthogonal(fsa, ws=FAKE + 1) == ALIGN
    need = fsa.fsa_orthogonalize_workspace_bytes(2, 64, 32, torch.float32)
    assert _orthogonal(fsa, n=need - 1) == WORKSPACE and _orthogonal(fsa, ws=None) == WORKSPACE
    assert _orthogonal(fsa, B=0, g=None, out=None, ws=None, n=0) == 0


def test_tensors_on_the_host_are_refused(fsa):
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    x, w = torch.ones(4, 8), torch.ones(8)
    for call in (lambda: fsa.fsa_norm_fwd(x, w), lambda: fsa.fsa_norm_bwd(x, None, x, w), lambda: fused_residual_norm(x, w, x),
                 lambda: fsa.fsa_gated_fwd(x, x, x, torch.ones(3, 4)), lambda: fused_gated_feed_forward(x, x, x, torch.ones(3, 4)),
                 lambda: fsa.fsa_gated_bwd(x, x, x, x, x), lambda: fsa.fsa_orthogonalize(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()

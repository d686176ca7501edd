"""The class losses without a GPU: the plan's arithmetic, workspace sizes and the C ABI's refusals."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # non-null, 16-byte aligned; never dereferenced on an error path


def test_the_plan_covers_every_tile_and_block(tmp_path):
    exe = str(tmp_path / "class_plan_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Xlinker", "--no-as-needed", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "native", "class_plan_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


@pytest.fixture(scope="module")
def fsa():
    from paper_2511_13645_amd import binding, build
    if build.is_stale():
        build.build_hip()
    return binding


def _fwd(fsa, **kw):
    a = dict(h=FAKE, hs=16, w=FAKE, ws=16, dt=0, T=8, V=10, D=16, scale=1.0, temp=1.0, ids=FAKE, logits=FAKE, lt=0, K=3, loss=FAKE,
             lse=FAKE, rg=FAKE, room=FAKE, bytes=0)
    a.update(kw)
    L = fsa.lib()
    if kw.get("xent"):
        return L.fsa_xent_fwd(*[a[n] for n in ("h", "hs", "w", "ws", "dt", "T", "V", "D", "scale", "ids", "loss", "lse", "rg", "room", "bytes")], None)
    return L.fsa_distill_fwd(*[a[n] for n in ("h", "hs", "w", "ws", "dt", "T", "V", "D", "scale", "temp", "ids", "logits", "lt", "K", "loss",
                                              "lse", "rg", "room", "bytes")], None)


def _bwd(fsa, **kw):
    a = dict(g=FAKE, h=FAKE, hs=16, w=FAKE, ws=16, dt=0, T=8, V=10, D=16, scale=1.0, ids=FAKE, lse=FAKE, rg=FAKE, gh=FAKE, gw=FAKE, room=FAKE,
             bytes=0)
    a.update(kw)
    return fsa.lib().fsa_xent_bwd(*[a[n] for n in ("g", "h", "hs", "w", "ws", "dt", "T", "V", "D", "scale", "ids", "lse", "rg", "gh", "gw",
                                                   "room", "bytes")], None)


def test_refusals(fsa):
    for name in ("h", "w", "ids", "logits", "loss", "lse"):
        assert _fwd(fsa, **{name: None}) == -1, name
    for kw in (dict(T=-1), dict(T=2 ** 23 + 1), dict(V=0), dict(V=2 ** 27 + 1), dict(D=0), dict(D=1025, hs=1025, ws=1025), dict(hs=15), dict(ws=15),
               dict(hs=2 ** 24 + 1), dict(K=0), dict(K=65), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(temp=0.0), dict(temp=float("inf")), dict(scale=1e-30, temp=1e30), dict(bytes=-1)):
        assert _fwd(fsa, **kw) == -2, kw
    assert _fwd(fsa, dt=3) == -3 and _fwd(fsa, lt=-1) == -3
    for kw in (dict(h=FAKE + 2), dict(w=FAKE + 1, dt=1), dict(ids=FAKE + 2), dict(logits=FAKE + 1, lt=2), dict(loss=FAKE + 1), dict(rg=FAKE + 2)):
        assert _fwd(fsa, **kw) == -4, kw
    need = fsa.lib().fsa_class_fwd_workspace_bytes(8, 10, 16, 0, 3, 1)
    assert need > 0 and _fwd(fsa, bytes=need - 1) == -7 and _fwd(fsa, room=None, bytes=need) == -7
    assert _fwd(fsa, room=FAKE + 8, bytes=need) == -4
    assert _fwd(fsa, T=0, h=None, ids=None, loss=None, lse=None) == 0         # nothing to do, nothing launched
    for name in ("g", "h", "w", "ids", "lse"):
        assert _bwd(fsa, **{name: None}) == -1, name
    assert _bwd(fsa, D=0) == -2 and _bwd(fsa, dt=9) == -3 and _bwd(fsa, gw=FAKE + 2) == -4 and _bwd(fsa, bytes=16) == -7
    assert "workspace" in fsa.status_string(-7)


def test_workspace_sizes(fsa):
    L = fsa.lib()
    for bad in ((-1, 10, 16, 0, 1), (8, 0, 16, 0, 1), (8, 10, 1025, 0, 1), (8, 10, 16, 5, 1), (8, 10, 16, 0, 65)):
        assert L.fsa_class_fwd_workspace_bytes(*bad, 1) == 0 and L.fsa_class_bwd_workspace_bytes(*bad, 1, 1) == 0
    for dt in (0, 1, 2):
        for D in (1, 128, 300):
            small = L.fsa_class_fwd_workspace_bytes(100, 5000, D, dt, 4, 0)
            assert 0 < small < L.fsa_class_fwd_workspace_bytes(100, 5000, D, dt, 4, 1)
            assert L.fsa_class_bwd_workspace_bytes(100, 5000, D, dt, 4, 0, 0) < L.fsa_class_bwd_workspace_bytes(100, 5000, D, dt, 4, 0, 1)

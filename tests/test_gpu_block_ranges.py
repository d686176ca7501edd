"""The block's operators at the ends of what they take: offsets beyond 32 bits, strides that no product reads in place, one table in two
places, gradients of sums and of shared and repeated leaves, both host paths, and a library that allocates nothing."""
import ctypes

import pytest
import torch

import block_bounds as bb
import test_gpu_block_orthogonal as ortho

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _normal(*shape, dtype=torch.float32, seed=0, unit=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0, unit, generator=gen)


def _plain(x, wg, wu, wd):
    return (torch.nn.functional.silu(x @ wg.T) * (x @ wu.T)) @ wd.T


def test_norm_beyond_32_bit_offsets():
    from paper_2511_13645_amd import binding as fsa
    t, d = 140_000, 16384
    assert t * d > 2 ** 31
    s, w = _normal(t, d, dtype=torch.bfloat16), _normal(d, seed=1)
    y, _ = fsa.fsa_norm_fwd(s, w)
    gx, gw = fsa.fsa_norm_bwd(y, None, s, w)
    rows = torch.tensor([0, 2 ** 31 // d - 1, 2 ** 31 // d, 2 ** 31 // d + 1, t - 1], device=DEV)
    want = bb.norm(s[rows], None, w, y[rows], None, 1e-6, s.dtype)
    bb.check("y", y[rows], *want["y"])
    bb.check("grad_x", gx[rows], *want["grad_x"])
    total, size = torch.zeros(2, d, dtype=torch.float64, device=DEV)
    for i in range(0, t, 10_000):
        u = s[i:i + 10_000].double()
        u = u * torch.rsqrt(u.pow(2).mean(1, keepdim=True) + 1e-6) * y[i:i + 10_000].double()
        total += u.sum(0)
        size += u.abs().sum(0)
    # a workgroup's rows, then the workgroups' parts, one after another: 137 rows and 1024 parts, and some 20 steps of a row
    bb.check("grad_weight", gw, total, (140 + 1024 + 20) * bb.V * size + bb.rounding(total, torch.float32))


@pytest.mark.parametrize("d,h", [(2048, 24), (16, 2048)])
def test_gated_rows_beyond_32_bit_offsets(d, h):
    """Of x, and of the hidden rows."""
    from paper_2511_13645_amd import binding as fsa
    t, o, dtype = 1_100_000, 16, torch.bfloat16
    assert t * max(d, h) > 2 ** 31
    x, wg, wu = _normal(t, d, dtype=dtype), _normal(h, d, dtype=dtype, seed=1, unit=d ** -0.5), _normal(h, d, dtype=dtype, seed=2, unit=d ** -0.5)
    wd, gy = _normal(o, h, dtype=dtype, seed=3, unit=h ** -0.5), _normal(t, o, dtype=dtype, seed=4)
    edge = 2 ** 31 // max(d, h)
    rows = torch.tensor([0, 1, edge - 1, edge, edge + 1, t - 1], device=DEV)
    want = bb.gated(x[rows], wg, wu, wd, gy[rows], "silu", dtype)
    y, kept = fsa.fsa_gated_fwd(x, wg, wu, wd, emit_kept=True)
    bb.check("y", y[rows], *want["y"])
    sums = None
    for given in (None, kept):
        gx, *grads = fsa.fsa_gated_bwd(gy, x, wg, wu, wd, given)
        bb.check("grad_x", gx[rows], *want["grad_x"])
        if sums is None:
            leaves = [v.double().requires_grad_(True) for v in (wg, wu, wd)]
            sums = [torch.zeros_like(v) for v in leaves]
            for i in range(0, t, 50_000):
                part = torch.autograd.grad(_plain(x[i:i + 50_000].double(), *leaves), leaves, gy[i:i + 50_000].double())
                for a, b in zip(sums, part):
                    a += b
        for got, total in zip(grads, sums):
            # of sums of either sign: a factor's rounding of half a step at most, by sqrt(3) less in the mean, and the result's
            assert (got.double() - total).norm().item() <= 2 * bb.HALF_STEP[dtype] * total.norm().item()


def test_orthogonalised_matrices_beyond_32_bit_offsets():
    from paper_2511_13645_amd import binding as fsa
    b, m, n = 2200, 16, 65536
    assert b * m * n > 2 ** 31
    g = _normal(b, m, n, dtype=torch.bfloat16)
    at = [0, 2 ** 31 // (m * n), b - 1]
    out = fsa.fsa_orthogonalize(g, ortho.ABC, 2)
    ortho._check(out[at], ortho._reference(g[at], [ortho.ABC] * 2), 2, g.dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_too_far_apart_for_a_product_to_read(dtype):
    from paper_2511_13645_amd import binding as fsa
    t, d, h, o = 70, 64, 72, 40
    far = (1 << 21) + 8
    x, wg, wu, wd, gy = (_normal(*s, seed=i).to(dtype) for i, s in enumerate(((t, d), (h, d), (h, d), (o, h), (t, o))))
    apart = []
    for v in (x, wg, wu, wd, gy):
        apart.append(torch.zeros(v.shape[0] * far, dtype=dtype, device=DEV).as_strided(v.shape, (far, 1)))
        apart[-1].copy_(v)
    xs, gs, us, ds, gys = apart
    assert torch.equal(fsa.fsa_gated_fwd(xs, gs, us, ds), fsa.fsa_gated_fwd(x, wg, wu, wd))
    assert all(torch.equal(a, b) for a, b in zip(fsa.fsa_gated_bwd(gys, xs, gs, us, ds), fsa.fsa_gated_bwd(gy, x, wg, wu, wd)))
    assert all(torch.equal(a, b) for a, b in zip(fsa.fsa_norm_fwd(xs, wg[0].clone(), xs), fsa.fsa_norm_fwd(x, wg[0].clone(), x)))
    assert torch.equal(fsa.fsa_orthogonalize(xs), fsa.fsa_orthogonalize(x))


def test_shared_leaves_and_gradients_of_sums():
    """One table as both, one tensor as rows and residual, and gradients that are one number repeated."""
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    x, w, wg, wd = (_normal(*s, seed=i).requires_grad_(True) for i, s in enumerate(((90, 48), (48,), (56, 48), (48, 56))))
    y, s = fused_residual_norm(x, w, x)
    got = torch.autograd.grad(fused_gated_feed_forward(y, wg, wg, wd).sum() + s.sum(), (x, w, wg, wd))
    leaves = [v.detach().double().requires_grad_(True) for v in (x, w, wg, wd)]
    a, b, c, e = leaves
    n = 2 * a * torch.rsqrt((2 * a).pow(2).mean(1, keepdim=True) + 1e-6) * b
    want = torch.autograd.grad(_plain(n, c, c, e).sum() + (2 * a).sum(), leaves)
    for p, q in zip(got, want):
        assert (p.double() - q).norm().item() <= 200 * bb.V * q.norm().item()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_both_host_paths_give_the_same(dtype, monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    fsa.lib()
    assert fsa._block_host is not None
    t, d, h = 130, 200, 96
    x, r, w, wg, wu, wd, g = (_normal(*s, seed=i, unit=0.3).to(dtype).requires_grad_(i < 6)
                              for i, s in enumerate(((t, d), (t, d), (d,), (h, d), (h, d), (d, h), (t, d))))

    def run():
        y, s = fused_residual_norm(x, w, r)
        z = fused_gated_feed_forward(y, wg, wu, wd, activation="gelu")
        q, same = fused_residual_norm(z, w)
        assert same is z
        return [y, s, z, q, *torch.autograd.grad((q, s), (x, r, w, wg, wu, wd), (g, g))]

    native = run()
    # no call of these is left to the Python code
    assert all(fsa._block_host.norm(x, w, residual, 1e-6) is not None for residual in (None, r))
    assert all(fsa._block_host.norm_fwd(x, w, residual, 1e-6) is not None for residual in (None, r))
    assert fsa._block_host.gated(x, wg, wu, wd, 1) is not None and fsa._block_host.gated_fwd(x, wg, wu, wd, 1) is not None
    monkeypatch.setattr(fsa, "_block_host", None)
    assert all(torch.equal(a, b) for a, b in zip(native, run()))


def test_second_derivatives_are_refused():
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    x, w, wg, wd = (_normal(*s, seed=i).requires_grad_(True) for i, s in enumerate(((20, 24), (24,), (32, 24), (24, 32))))
    for y in (fused_residual_norm(x, w)[0], fused_gated_feed_forward(x, wg, wg, wd)):
        # (as with torch's own functions that are differentiable once: of a gradient that itself wants one)
        g = torch.autograd.grad(y, x, torch.ones_like(y).requires_grad_(True), create_graph=True)[0]
        with pytest.raises(RuntimeError, match="differentiable once|once_differentiable"):
            g.sum().backward()


def test_the_library_allocates_nothing():
    from paper_2511_13645_amd import binding as fsa
    t, d, h = 300, 136, 264
    x, w, wg, wu, wd = (_normal(*s, seed=i) for i, s in enumerate(((t, d), (d,), (h, d), (h, d), (d, h))))
    y, s, gx, gw, gg, gu, gd, out, gs = (torch.empty_like(v) for v in (x, x, x, w, wg, wu, wd, wg, x))
    L, st = fsa.lib(), torch.cuda.current_stream().cuda_stream
    kept = torch.empty(fsa.lib().fsa_gated_kept_bytes(t, d, h, d, 0), dtype=torch.uint8, device=DEV)
    ws = torch.empty(max(fsa.fsa_gated_bwd_workspace_bytes(t, d, h, d, x.dtype), fsa.fsa_gated_fwd_workspace_bytes(t, d, h, d, x.dtype),
                         fsa.fsa_norm_bwd_workspace_bytes(t, d, x.dtype), fsa.fsa_orthogonalize_workspace_bytes(1, h, d, x.dtype)),
                     dtype=torch.uint8, device=DEV)
    P = lambda v: v.data_ptr()
    operands = (P(x), d, P(wg), d, P(wu), d, P(wd), h, 0, 0, t, d, h, d)
    triples = (ctypes.c_float * 6)(*fsa.ORTHOGONAL_COEFFICIENTS * 2)
    call = lambda: (L.fsa_norm_fwd(P(x), d, P(x), d, P(w), 0, 0, t, d, 1e-6, P(y), P(s), st) or
                    L.fsa_gated_fwd(*operands, P(y), P(kept), P(ws), ws.numel(), st) or
                    L.fsa_gated_bwd(P(y), d, *operands, P(kept), P(gx), P(gg), P(gu), P(gd), P(ws), ws.numel(), st) or
                    L.fsa_norm_bwd(P(gx), P(y), P(s), d, P(w), 0, 0, t, d, 1e-6, P(gs), P(gw), P(ws), ws.numel(), st) or
                    L.fsa_orthogonalize(P(gg), 0, d, 0, 1, h, d, triples, 2, 1e-7, 1.0, P(out), P(ws), ws.numel(), st))
    assert call() == 0
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()
    for _ in range(3):
        assert call() == 0
    torch.cuda.synchronize()
    assert (torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()) == before

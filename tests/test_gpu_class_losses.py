"""Softmax cross entropy and distillation over many classes against their definition in 64 bits: every type, rows from
none to several tiles, classes from one up, odd depths, holes and rows without a slot, strides, gradients alone."""
import math

import pytest
import torch

from class_util import DTYPES, bounds, check, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fsa():
    from paper_2511_13645_amd import binding
    binding.lib()
    return binding


def forward(fsa, op, h, w, ids, logits, temperature, scale, **kw):
    if op == "xent":
        return fsa.fsa_xent_fwd(h, w, ids, scale, **kw)
    return fsa.fsa_distill_fwd(h, w, ids, logits, temperature, scale, **kw)


def backward(fsa, op, g, h, w, ids, logits, lse, row_grad, temperature, scale, **kw):
    if op == "xent":
        return fsa.fsa_xent_bwd(g, h, w, ids, lse, row_grad, scale, **kw)
    return fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, temperature, scale, **kw)


def compare(fsa, op, dtype, h, w, ids, logits, g, temperature=1.0, scale=1.0):
    """Forward and backward against the definition; returns what they gave."""
    ref, x = reference(h, w, ids, logits, temperature, scale, g)
    lim = bounds(dtype, x, g)
    loss, lse, row_grad = forward(fsa, op, h, w, ids, logits, temperature, scale, emit_row_grad=True)
    alone, lse_alone, none = forward(fsa, op, h, w, ids, logits, temperature, scale)
    assert none is None
    grad_h, grad_w = backward(fsa, op, g, h, w, ids, logits, lse, row_grad, temperature, scale)
    assert grad_h.dtype == h.dtype and grad_w.dtype == w.dtype
    for name, got, d in (("loss", loss, "f32"), ("lse", lse, "f32"), ("row_grad", row_grad, "f32"), ("grad_h", grad_h, dtype),
                         ("grad_w", grad_w, dtype)):
        check(got, ref[name], lim[name], d, name)
    check(alone, ref["loss"], lim["loss"], "f32", "loss alone")
    check(lse_alone, ref["lse"], lim["lse"], "f32", "lse alone")
    return loss, lse, row_grad, grad_h, grad_w


SIZES = [(1, 1, 1), (1, 47, 128), (2, 33, 3), (5, 1000, 64), (31, 64, 100), (32, 32, 32), (33, 129, 65), (64, 31, 128),
         (65, 4097, 37), (127, 500, 256), (128, 2, 255), (129, 96, 129), (200, 3001, 96), (300, 65, 200), (513, 129, 16),
         (1, 1, 257), (33, 700, 602), (70, 95, 384), (65, 33, 1024), (129, 257, 640), (40, 1500, 385)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_cross_entropy(fsa, dtype, T, V, D):
    h, w, ids, _, g = inputs("xent", dtype, T, V, D, seed=T + V + D)
    compare(fsa, "xent", dtype, h, w, ids, None, g, scale=0.75)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,K", [(1, 1, 8, 1), (3, 70, 20, 64), (40, 64, 64, 64), (65, 1000, 100, 10), (130, 2049, 128, 33),
                                     (257, 200, 250, 5), (1, 5000, 128, 17), (70, 300, 602, 50), (33, 64, 300, 64), (65, 40, 1001, 3)])
def test_distillation(fsa, dtype, T, V, D, K):
    h, w, ids, logits, g = inputs("distill", dtype, T, V, D, K, seed=T + V + K)
    compare(fsa, "distill", dtype, h, w, ids, logits, g, temperature=2.0, scale=1.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [96, 602])
def test_rows_without_a_slot_hold_anything(fsa, dtype, D):
    """NaN, infinities and the type's largest values in rows without a slot reach no other row, no class and no result."""
    T, V, K = 70, 300, 5
    h, w, ids, logits, g = inputs("distill", dtype, T, V, D, K, seed=3)
    dead = torch.zeros(T, dtype=torch.bool, device=h.device)
    dead[torch.tensor([0, 5, 31, 32, 33, 64, 69])] = True
    ids[dead] = -1
    clean = compare(fsa, "distill", dtype, h, w, ids, logits, g, 1.0, 1.0)
    h2, g2, logits2 = h.clone(), g.clone(), logits.clone()
    h2[0], h2[5], h2[31], h2[32] = math.nan, math.inf, -math.inf, torch.finfo(h.dtype).max
    h2[33], h2[64], h2[69] = torch.finfo(h.dtype).min, math.nan, 1e4
    g2[dead] = torch.tensor([math.nan, math.inf, -math.inf, 3e38, 1e30, -3e38, math.nan], device=g.device)
    logits2[ids < 0] = math.nan                          # also in empty slots of rows that have others
    lse2 = clean[1].clone()
    loss, lse, rg = fsa.fsa_distill_fwd(h2, w, ids, logits2, 1.0, 1.0, emit_row_grad=True)
    lse2[dead] = math.nan
    rg2 = rg.clone()
    rg2[dead] = math.nan
    gh, gw = fsa.fsa_distill_bwd(g2, h2, w, ids, logits2, lse2, rg2, 1.0, 1.0)
    for a, b, name in zip((loss, lse, rg, gh, gw), clean, ("loss", "lse", "row_grad", "grad_h", "grad_w")):
        assert torch.equal(a, b), name
    assert float(loss[dead].abs().sum()) == 0 and float(gh[dead].abs().sum()) == 0 and float(lse[dead].abs().sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 300])
def test_no_row_has_a_slot(fsa, dtype, D):
    h, w, ids, _, g = inputs("xent", dtype, 40, 77, D)
    ids.fill_(-5)
    h.fill_(math.nan)
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    gh, gw = fsa.fsa_xent_bwd(g, h, w, ids, lse, rg)
    for t in (loss, lse, rg, gh, gw):
        assert float(t.abs().sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_teacher_logits_of_no_weight(fsa, dtype):
    """-inf is a weight of nothing, the type's lowest value beside others too, and a row of only that is uniform."""
    h, w, ids, logits, g = inputs("distill", dtype, 12, 90, 64, 8, holes=False)
    lowest = torch.finfo(logits.dtype).min
    logits[0, 1:] = -math.inf
    logits[1] = -math.inf                                # a row without any weight: as one without slots
    logits[2] = lowest
    logits[3, 2:] = lowest
    logits[4, ::2] = -math.inf
    got = compare(fsa, "distill", dtype, h, w, ids, logits, g)
    assert float(got[0][1]) == 0 and float(got[3][1].abs().sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [100, 390])
def test_classes_that_are_not_there(fsa, dtype, D):
    """An ID of V or more is not read: NaN in its row's loss, and the row's gradient is the softmax's alone."""
    h, w, ids, _, g = inputs("xent", dtype, 37, 50, D, holes=False)
    ids[7], ids[36] = 50, 2 ** 31 - 1
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    assert torch.isnan(loss[[7, 36]]).all() and int(torch.isnan(loss).sum()) == 2 and bool(torch.isfinite(lse).all())
    gh, gw = fsa.fsa_xent_bwd(g, h, w, ids, lse, rg)
    p = (h.double() @ w.double().T - lse.double()[:, None]).exp()
    rows = torch.arange(37, device=h.device)
    keep = (rows != 7) & (rows != 36)
    q = torch.zeros_like(p)
    q[rows[keep], ids[keep].long()] = 1.0
    d = g.double()[:, None] * (p - q)
    _, x = reference(h, w, ids.clamp(max=49), g=g)
    lim = bounds(dtype, x, g)
    check(gh, d @ w.double(), lim["grad_h"], dtype, "grad_h")
    check(gw, d.T @ h.double(), lim["grad_w"], dtype, "grad_w")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [128, 500])
def test_one_class_named_twice_counts_twice(fsa, dtype, D):
    h, w, ids, logits, g = inputs("distill", dtype, 33, 60, D, 6, holes=False)
    ids[:, 3] = ids[:, 0]
    ids[::2, 5] = ids[::2, 0]
    compare(fsa, "distill", dtype, h, w, ids, logits, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 448])
@pytest.mark.parametrize("spread", [1e-3, 40.0])
def test_flat_and_peaked_scores(fsa, dtype, D, spread):
    """Scores all alike, and scores of hundreds, whose running maximum moves again and again."""
    h, w, ids, _, g = inputs("xent", dtype, 65, 700, D, seed=5, spread=spread)
    compare(fsa, "xent", dtype, h, w, ids, None, g)


def test_rows_and_classes_of_very_different_size(fsa):
    """fp32: elements 2^-20 below their table's largest keep their share of the results."""
    h, w, ids, _, g = inputs("xent", "f32", 64, 500, 100, seed=8)
    w[::3] *= 2.0 ** -12
    w[1] *= 2.0 ** 6
    h[::2] *= 2.0 ** -10
    h[3] *= 2.0 ** 3
    g[::4] *= 1e-4
    compare(fsa, "xent", "f32", h, w, ids, None, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [33, 128, 601])
def test_strides_and_alignment(fsa, dtype, D):
    """Rows apart, off the 16-byte grid, and columns of a wider matrix: as the same rows by themselves, to the last bit
    where neither is laid out anew."""
    T, V = 300, 1100
    h, w, ids, _, g = inputs("xent", dtype, T, V, D)
    want = compare(fsa, "xent", dtype, h, w, ids, None, g)
    big_h = torch.full((T + 1, D + 7), math.nan, dtype=h.dtype, device=h.device)
    big_w = torch.full((V + 1, D + 5), math.nan, dtype=h.dtype, device=h.device)
    vh, vw = big_h[1:, 3:3 + D], big_w[1:, 1:1 + D]
    vh.copy_(h)
    vw.copy_(w)
    got = compare(fsa, "xent", dtype, vh, vw, ids, None, g)
    for a, b in zip(got, want):
        assert a.shape == b.shape and a.is_contiguous()
        assert torch.equal(a, b) or D == 128             # (a whole depth on the grid is streamed as it is)


@pytest.mark.parametrize("op", ["xent", "distill"])
@pytest.mark.parametrize("D", [64, 320])
def test_gradients_apart_and_again(fsa, op, D):
    """Either gradient alone, and grad_h without what the forward saved, are the same bits; twice as well."""
    h, w, ids, logits, g = inputs(op, "bf16", 130, 513, D, 4)
    loss, lse, rg = forward(fsa, op, h, w, ids, logits, 1.0, 1.0, emit_row_grad=True)
    again = forward(fsa, op, h, w, ids, logits, 1.0, 1.0, emit_row_grad=True)
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, rg), again))
    both = backward(fsa, op, g, h, w, ids, logits, lse, rg, 1.0, 1.0)
    only_h = backward(fsa, op, g, h, w, ids, logits, lse, rg, 1.0, 1.0, want_w=False)
    only_w = backward(fsa, op, g, h, w, ids, logits, lse, rg, 1.0, 1.0, want_h=False)
    fresh = backward(fsa, op, g, h, w, ids, logits, lse, None, 1.0, 1.0)
    assert only_h[1] is None and only_w[0] is None
    assert torch.equal(only_h[0], both[0]) and torch.equal(only_w[1], both[1])
    assert torch.equal(fresh[0], both[0]) and torch.equal(fresh[1], both[1])


@pytest.mark.parametrize("D", [40, 512])
def test_no_rows(fsa, D):
    h, w, ids, _, g = inputs("xent", "f32", 0, 9, D)
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    gh, gw = fsa.fsa_xent_bwd(g, h, w, ids, lse, rg)
    assert loss.shape == (0,) and gh.shape == (0, D) and gw.shape == (9, D) and float(gw.abs().sum()) == 0


@pytest.mark.parametrize("op", ["xent", "distill"])
@pytest.mark.parametrize("D", [24, 280])
def test_gradients_against_differences(fsa, op, D):
    """Losses at h +- e d and w +- e d: their difference over 2e is the gradient along d, off by e^2 / 6 of the third
    derivative (at most 8 a^3 for scores that move by a along d) and by the losses' rounding over e."""
    h, w, ids, logits, g = inputs(op, "f32", 48, 150, D, 6, seed=2)
    loss, lse, rg = forward(fsa, op, h, w, ids, logits, 1.0, 1.0, emit_row_grad=True)
    gh, gw = backward(fsa, op, g, h, w, ids, logits, lse, rg, 1.0, 1.0)
    gen = torch.Generator().manual_seed(1)
    e = 2.0 ** -7
    for t, grad, other in ((h, gh, w), (w, gw, h)):
        d = torch.randn(t.shape, generator=gen).to(t.device)
        d /= (d @ other.T).abs().max()                   # scores move by at most 1 along d
        ends = []
        for sign in (1.0, -1.0):
            a, b = (t + sign * e * d, w) if t is h else (h, t + sign * e * d)
            ends.append(forward(fsa, op, a, b, ids, logits, 1.0, 1.0)[0].double())
        slope = (ends[0] - ends[1]) / (2 * e)
        want = float((g.double() * slope).sum())
        live = float((g.abs() * (loss != 0)).sum())
        tol = live * (8 * e * e / 6 + 2 * 2.0 ** -20 / (2 * e) * (float(lse.abs().max()) + 16) / 16)
        assert abs(float((grad.double() * d.double()).sum()) - want) <= tol


def test_autograd(fsa):
    from paper_2511_13645_amd.autograd import fused_cross_entropy, fused_distillation
    h, w, ids, _, g = inputs("xent", "f32", 70, 200, 64)
    h.requires_grad_(True)
    w.requires_grad_(True)
    a, b = torch.autograd.grad((fused_cross_entropy(h, w, ids, scale=0.5) * g).sum(), (h, w))
    loss, lse, rg = fsa.fsa_xent_fwd(h.detach(), w.detach(), ids, 0.5, emit_row_grad=True)
    c, d = fsa.fsa_xent_bwd(g, h.detach(), w.detach(), ids, lse, rg, 0.5)
    assert torch.equal(a, c) and torch.equal(b, d)
    fused_cross_entropy(h, w, ids, scale=0.5).sum().backward()          # an expanded gradient
    ones = fsa.fsa_xent_bwd(torch.ones_like(g), h.detach(), w.detach(), ids, lse, rg, 0.5)
    assert torch.equal(h.grad, ones[0]) and torch.equal(w.grad, ones[1])
    with torch.no_grad():
        quiet = fused_cross_entropy(h, w, ids, scale=0.5)
    assert not quiet.requires_grad and torch.equal(quiet, fsa.fsa_xent_fwd(h.detach(), w.detach(), ids, 0.5)[0])
    only_w = fused_cross_entropy(h.detach(), w, ids, scale=0.5)
    assert torch.equal(torch.autograd.grad(only_w, w, g)[0], d)
    k, ids2, logits = 5, *inputs("distill", "f32", 70, 200, 64, 5)[2:4]
    l2 = fused_distillation(h, w, ids2, logits, temperature=2.0)
    e, f = torch.autograd.grad(l2, (h, w), g, retain_graph=True)
    loss, lse, rg = fsa.fsa_distill_fwd(h.detach(), w.detach(), ids2, logits, 2.0, emit_row_grad=True)
    x, y = fsa.fsa_distill_bwd(g, h.detach(), w.detach(), ids2, logits, lse, rg, 2.0)
    assert torch.equal(e, x) and torch.equal(f, y) and torch.equal(l2.detach(), loss)
    gg = g.clone().requires_grad_(True)
    once = torch.autograd.grad(l2, h, gg, create_graph=True)[0]
    with pytest.raises(RuntimeError):
        once.sum().backward()


def test_native_and_python_paths_agree(fsa, monkeypatch):
    """The native host path answers as the Python binding, bit for bit, and refuses what that refuses."""
    from paper_2511_13645_amd import autograd
    h, w, ids, logits, g = inputs("distill", "bf16", 100, 300, 96, 7)
    h.requires_grad_(True)
    w.requires_grad_(True)

    def run():
        f = fsa.fsa_distill_fwd(h.detach(), w.detach(), ids, logits, 2.0, emit_row_grad=True)
        loss = autograd.fused_distillation(h, w, ids, logits, temperature=2.0)
        return (*f, loss.detach(), *torch.autograd.grad(loss, (h, w), g))
    assert fsa._class_host is not None
    native = run()
    monkeypatch.setattr(fsa, "_class_host", None)
    plain = run()
    assert all(torch.equal(a, b) for a, b in zip(native, plain))


def test_wrong_arguments_are_refused(fsa):
    from paper_2511_13645_amd.autograd import fused_cross_entropy
    h, w, ids, logits, g = inputs("distill", "f32", 6, 20, 16, 3)
    y = ids[:, 0].contiguous()
    for bad in ((h.half(), w, y), (h, w, y.long()), (h.double(), w.double(), y)):
        with pytest.raises(TypeError):
            fused_cross_entropy(*bad)
    for bad in ((h, w[:, :8], y), (h, w, y[:5]), (h.cpu(), w, y), (h, w, ids), (h.T, w, y), (h.expand(2, 6, 16), w, y),
                (h[:1].expand(6, 16), w, y), (h, w, y.cpu())):
        with pytest.raises(ValueError):
            fused_cross_entropy(*bad)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan)):
        with pytest.raises(fsa.FsaError):
            fused_cross_entropy(h, w, y, **kw)
    with pytest.raises(fsa.FsaError):
        fsa.fsa_distill_fwd(h, w, ids, logits, 0.0)
    many = torch.zeros((6, 65), dtype=torch.int32, device=h.device)
    with pytest.raises(fsa.FsaError):
        fsa.fsa_distill_fwd(h, w, many, many.float())
    with pytest.raises(ValueError):
        fsa.fsa_distill_fwd(h, w, ids, logits[:, :2])
    with pytest.raises(fsa.FsaError):
        fsa.fsa_xent_fwd(torch.zeros((2, 1025), device=h.device), torch.zeros((3, 1025), device=h.device), y[:2].contiguous())
    small = torch.empty(16, dtype=torch.uint8, device=h.device)
    with pytest.raises(fsa.FsaError):
        fsa.fsa_xent_fwd(h, w, y, workspace=small)
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, y, emit_row_grad=True)
    with pytest.raises(fsa.FsaError):
        fsa.fsa_xent_bwd(g, h, w, y, lse, rg, workspace=small)
    with pytest.raises(ValueError):
        fsa.fsa_xent_bwd(g[:3], h, w, y, lse, rg)
    with pytest.raises(ValueError):
        fsa.fsa_xent_bwd(g, h, w, y, lse, rg[:, :4])


@pytest.mark.parametrize("D", [128, 384])
def test_another_stream_and_a_graph(fsa, D):
    """On a stream of its own, and captured with the caller's workspace: every replay reads what its inputs hold then."""
    h, w, ids, _, g = inputs("xent", "f16", 200, 3000, D)
    want = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    grads = fsa.fsa_xent_bwd(g, h, w, ids, want[1], want[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True, stream=side)
    back = fsa.fsa_xent_bwd(g, h, w, ids, got[1], got[2], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *back), (*want, *grads)))
    room = max(fsa.fsa_class_fwd_workspace_bytes(200, 3000, D, h.dtype, 1, True), fsa.fsa_class_bwd_workspace_bytes(200, 3000, D, h.dtype))
    ws = torch.empty(room, dtype=torch.uint8, device=h.device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True, workspace=ws)
        b = fsa.fsa_xent_bwd(g, h, w, ids, f[1], f[2], workspace=ws)
    for turn in range(3):
        h.mul_(0.5)
        ids.copy_(ids.roll(turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
        grads = fsa.fsa_xent_bwd(g, h, w, ids, want[1], want[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((*f, *b), (*want, *grads)))


def test_the_library_allocates_nothing(fsa):
    h, w, ids, _, g = inputs("xent", "bf16", 64, 500, 128)
    L, st = fsa.lib(), torch.cuda.current_stream().cuda_stream
    f32 = dict(dtype=torch.float32, device=h.device)
    loss, lse, rg = torch.empty(64, **f32), torch.empty(64, **f32), torch.empty((64, 128), **f32)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(max(fsa.fsa_class_fwd_workspace_bytes(64, 500, 128, h.dtype, 1, True),
                         fsa.fsa_class_bwd_workspace_bytes(64, 500, 128, h.dtype)), dtype=torch.uint8, device=h.device)
    P = lambda t: t.data_ptr()
    call = lambda: (L.fsa_xent_fwd(P(h), 128, P(w), 128, 1, 64, 500, 128, 1.0, P(ids), P(loss), P(lse), P(rg), P(ws), ws.numel(), st) or
                    L.fsa_xent_bwd(P(g), P(h), 128, P(w), 128, 1, 64, 500, 128, 1.0, P(ids), P(lse), P(rg), P(gh), P(gw), P(ws),
                                   ws.numel(), st))
    assert call() == 0
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()
    for _ in range(3):
        assert call() == 0
    torch.cuda.synchronize()
    assert (torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()) == before


@pytest.mark.parametrize("D,V", [(128, 17_000_000), (1024, 2_200_000)])
def test_tables_beyond_32_bit_offsets(fsa, D, V):
    """More than 2^31 elements: the table's first and last classes, and some between, in losses and gradients."""
    T = 5
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda:0").normal_(0, 1.0 / math.sqrt(D), generator=gen)
    h = torch.randn((T, D), generator=gen, device="cuda:0").bfloat16()
    ids = torch.tensor([0, V - 1, V // 2, 2 ** 31 // D, -1], dtype=torch.int32, device="cuda:0")
    g = torch.tensor([1.0, -2.0, 0.5, 3.0, 1.0], device="cuda:0")
    loss, lse, rg = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True)
    gh, gw = fsa.fsa_xent_bwd(g, h, w, ids, lse, rg)
    total, mean = torch.zeros(T, dtype=torch.float64, device="cuda:0"), torch.zeros((T, D), dtype=torch.float64, device="cuda:0")
    step = 1 << 18
    for a in range(0, V, step):
        e = (h.double() @ w[a:a + step].double().T).exp()
        total += e.sum(1)
        mean += e @ w[a:a + step].double()
    want = total.log()
    live = ids >= 0
    y = ids.clamp(min=0).long()
    z = (h.double() * w[y].double()).sum(1)
    assert float((lse - want)[live].abs().max()) < 1e-5 and float((loss - (want - z))[live].abs().max()) < 2e-5
    row = g.double()[:, None] * (mean / total[:, None] - w[y].double())
    check(gh[live], row[live], (2.0 ** -8 * g.double().abs()[:, None] * (w[y].double().abs() + 1e-3))[live], "bf16", "grad_h")
    rows = torch.cat([y[live], torch.tensor([1, V - 2, 2 ** 31 // D + 1], device="cuda:0")])
    p = (h.double() @ w[rows].double().T - want[:, None]).exp()
    d = (p - (rows[None, :] == ids[:, None]).double()) * torch.where(live, g.double(), 0.0)[:, None]
    bound = 2 * 2.0 ** -8 * (d.abs().T @ h.double().abs())
    check(gw[rows], d.T @ h.double(), bound, "bf16", "grad_w")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [80, 400])
def test_rows_that_the_teacher_gives_nothing_hold_anything(fsa, dtype, D):
    """A row whose slots all have logits of -inf is as one without slots: what it holds does not move another's units."""
    h, w, ids, logits, g = inputs("distill", dtype, 40, 120, D, 4, holes=False)
    dead = torch.zeros(40, dtype=torch.bool, device=h.device)
    dead[[3, 33]] = True
    logits[dead] = -math.inf
    want = compare(fsa, "distill", dtype, h, w, ids, logits, g)
    h[3], h[33] = torch.finfo(h.dtype).max, math.nan
    g[3], g[33] = 3e38, math.nan
    loss, lse, rg = fsa.fsa_distill_fwd(h, w, ids, logits, emit_row_grad=True)
    gh, gw = fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, rg)
    for a, b, name in zip((loss, lse, rg, gh, gw), want, ("loss", "lse", "row_grad", "grad_h", "grad_w")):
        assert torch.equal(a, b), name

"""Captured backwards of the block that the Python code makes (of tensors that the native host path leaves to it, or without that path):
as the native ones, refused beside an eager graph of the same leaves, and right without."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _calls():
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    gen = torch.Generator(device=DEV).manual_seed(0)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV).requires_grad_(True)
    x, r, w, wg, wu, wd = n(50, 32), n(50, 32), n(32), n(48, 32), n(48, 32), n(32, 48)
    return x, n(50, 32).detach(), (lambda: fused_gated_feed_forward(x, wg, wu, wd), lambda: fused_residual_norm(x, w, r)[0])


def _capture(call, x, g):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = torch.autograd.grad(call(), (x,), g)[0]
    return graph, out


def test_beside_an_eager_graph(monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    fsa.lib()
    assert fsa._block_host is not None
    monkeypatch.setattr(fsa, "norm", lambda *a: None)
    monkeypatch.setattr(fsa, "gated", lambda *a: None)
    x, g, calls = _calls()
    for call in calls:
        eager = call()
        assert "Backward" in type(eager.grad_fn).__name__ and hasattr(eager.grad_fn, "needs_input_grad")     # Python's own function
        want = torch.autograd.grad(call(), (x,), g)[0]
        torch.cuda.synchronize()
        with pytest.raises(RuntimeError, match="eager graph"):
            _capture(call, x, g)
        torch.cuda.synchronize()
        del eager
        graph, got = _capture(call, x, g)
        for _ in range(3):
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)


@pytest.mark.parametrize("python", [False, True])
def test_beside_an_eager_graph_of_what_a_cast_is_made_of(python, monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward, fused_residual_norm
    fsa.lib()
    assert fsa._block_host is not None
    if python:
        monkeypatch.setattr(fsa, "norm", lambda *a: None)
        monkeypatch.setattr(fsa, "gated", lambda *a: None)
    gen = torch.Generator(device=DEV).manual_seed(0)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    x, g, both, wd = n(50, 32).bfloat16(), n(50, 32).bfloat16(), n(96, 32).requires_grad_(True), n(32, 48).requires_grad_(True)
    w = n(32).requires_grad_(True)

    def gated():
        tables = both.bfloat16()
        return fused_gated_feed_forward(x, tables[:48], tables[48:], wd.bfloat16())

    for call, leaves in ((gated, (both, wd)), (lambda: fused_residual_norm(x, w.bfloat16())[0], (w,))):
        eager = call()
        want = torch.autograd.grad(call(), leaves, g)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="eager graph"):
            with torch.cuda.graph(graph):
                torch.autograd.grad(call(), leaves, g)
        torch.cuda.synchronize()
        del eager
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = torch.autograd.grad(call(), leaves, g)
        for _ in range(3):
            for v in got:
                v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_without_the_native_host_path(monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    fsa.lib()
    monkeypatch.setattr(fsa, "_block_host", None)
    x, g, calls = _calls()
    for call in calls:
        with pytest.raises(RuntimeError, match="without the native host path"):
            _capture(call, x, g)
        torch.cuda.synchronize()
        y = call()                                           # a forward alone is captured, and eager backwards run
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            z = call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, z)
        torch.autograd.grad(y, (x,), g)

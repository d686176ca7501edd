"""A captured backward of the block that the Python code makes without the native host path: refused where its gradients go to leaves.  No
GPU: that a capture is under way is what the test says."""
import pytest
import torch


class _Twice(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x):
        return x * 2

    @staticmethod
    def backward(ctx, g):
        from paper_2511_13645_amd import binding
        binding.refuse_capture("a test")
        return g * 2


def test_without_the_native_host_path(monkeypatch):
    from paper_2511_13645_amd import binding
    monkeypatch.setattr(binding, "_block_host", None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    x = torch.ones(3, requires_grad=True)
    run = lambda v: torch.autograd.grad(_Twice.apply(v).sum(), x)[0]
    assert torch.equal(run(x), torch.full((3,), 2.0))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="a test cannot be captured without the native host path"):
        run(x)
    for view in (lambda: x.double(), lambda: x.view(3, 1), lambda: x.half().float()[:2]):
        with pytest.raises(RuntimeError, match="a test cannot be captured without the native host path"):
            run(view())
    assert torch.equal(run(x * x), torch.full((3,), 4.0))


def test_both_functions_ask(monkeypatch):
    from paper_2511_13645_amd import autograd, binding
    asked = []

    def refuse(what):
        asked.append(what)
        raise RuntimeError(what)

    monkeypatch.setattr(binding, "refuse_capture", refuse)
    x, w = torch.ones((4, 8), requires_grad=True), torch.ones((8, 8))
    monkeypatch.setattr(binding, "fsa_norm_fwd", lambda x, w, r, eps: (x.detach() * 1, None))
    monkeypatch.setattr(binding, "fsa_gated_fwd", lambda x, *a, **k: x.detach() * 1)
    for y in (autograd._ResidualNorm.apply(x, w[0], None, 1e-6), autograd._GatedFeedForward.apply(x, w, w, w, "silu", False, False)):
        with pytest.raises(RuntimeError):
            y.sum().backward()
    assert asked == ["a norm", "a gated block"]

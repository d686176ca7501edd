"""Class losses with a stream given: what the call allocates is that stream's own."""
import pytest
import torch

from class_util import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fsa():
    from paper_2511_13645_amd import binding
    binding.lib()
    return binding


def calls(fsa, op, h, w, ids, logits, g, **kw):
    if op == "xent":
        loss, lse, row_grad = fsa.fsa_xent_fwd(h, w, ids, emit_row_grad=True, **kw)
        return (loss, lse, row_grad, *fsa.fsa_xent_bwd(g, h, w, ids, lse, row_grad, **kw))
    loss, lse, row_grad = fsa.fsa_distill_fwd(h, w, ids, logits, emit_row_grad=True, **kw)
    return (loss, lse, row_grad, *fsa.fsa_distill_bwd(g, h, w, ids, logits, lse, row_grad, **kw))


@pytest.mark.parametrize("op", ["xent", "distill"])
def test_results_and_workspace_are_the_streams(fsa, op, monkeypatch):
    """Every allocation of a call with a stream is made with that stream current, results and workspace alike."""
    args = inputs(op, "bf16", 130, 700, 96, 5)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    made, empty, like = [], torch.empty, torch.empty_like
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(torch.cuda.current_stream()) or empty(*a, **k))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: made.append(torch.cuda.current_stream()) or like(*a, **k))
    calls(fsa, op, *args, stream=side)
    monkeypatch.undo()
    assert len(made) == 7 and all(s == side for s in made)      # three results and two gradients, a workspace each way
    assert torch.cuda.current_stream() != side
    torch.cuda.synchronize()


@pytest.mark.parametrize("op", ["xent", "distill"])
@pytest.mark.parametrize("D", [96, 320])
def test_calls_on_two_streams_at_a_time(fsa, op, D):
    """Calls on the current stream and on another one right after each other, their workspaces and what else is dropped free
    to be given out again: neither writes what the other works on."""
    a, b = inputs(op, "f16", 300, 5000, D, 5, seed=1), inputs(op, "f16", 260, 5000, D, 5, seed=2)
    want_a, want_b = calls(fsa, op, *a), calls(fsa, op, *b)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for _ in range(3):
            got.append((calls(fsa, op, *a)[3:], want_a[3:]))            # loss, lse and row_grad dropped
            got.append((calls(fsa, op, *b, stream=side)[3:], want_b[3:]))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, w in got for x, y in zip(g, w))

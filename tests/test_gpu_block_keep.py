"""What a gated block's forward keeps for its backward, as the caller chooses it, and where there is no room for it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, D, H, O = 20000, 512, 2048, 64                           # sizes that keep by themselves: 0.33 GB


def _leaves(dtype=torch.bfloat16):
    gen = torch.Generator(device=DEV).manual_seed(0)
    n = lambda *s: torch.randn(s, generator=gen, device=DEV)
    return [v.to(dtype).requires_grad_(True) for v in (n(T, D), n(H, D) * D ** -0.5, n(H, D) * D ** -0.5, n(O, H) * H ** -0.5)], n(T, O).to(dtype)


def _held(call):
    """The call's result and the bytes that it and its graph hold."""
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = call()
    return y, torch.cuda.memory_allocated() - before - y.numel() * y.element_size()


@pytest.fixture(params=["native", "python"])
def block(request, monkeypatch):
    from paper_2511_13645_amd import binding as fsa
    from paper_2511_13645_amd.autograd import fused_gated_feed_forward
    fsa.lib()
    assert fsa._block_host is not None
    if request.param == "python":
        monkeypatch.setattr(fsa, "_block_host", None)
    return fused_gated_feed_forward


def test_kept_or_made_again(block):
    from paper_2511_13645_amd import binding as fsa
    leaves, gy = _leaves()
    size = fsa.lib().fsa_gated_kept_bytes(T, D, H, O, 1)
    assert size >= T * H * 8 and fsa.fsa_gated_keep_pays(T, D, H, O, torch.bfloat16)
    grads = {}
    for keep in (None, True, False):
        y, held = _held(lambda: block(*leaves, keep=keep))
        assert held < size // 100 if keep is False else size <= held < size * 1.01, keep
        grads[keep] = torch.autograd.grad(y, leaves, gy)
        del y
    assert all(torch.equal(a, b) for a, b in zip(grads[None], grads[True]))
    # each is off by its own rounding and a factor's, 2^-8 by sqrt(3) in the mean square at most: by twice sqrt(2 / 3) 2^-8 from one another
    for a, b in zip(grads[True], grads[False]):
        assert (a.double() - b.double()).norm().item() <= 1.64 * 2.0 ** -8 * b.double().norm().item()


def test_where_it_would_not_pay(block):
    leaves, gy = _leaves()
    small = [leaves[0].detach()[:, :64].contiguous().requires_grad_(True)] + [v.detach()[:, :64].contiguous().requires_grad_(True) for v in leaves[1:3]] + leaves[3:]
    assert _held(lambda: block(*small))[1] < 1 << 20 < T * H * 8 <= _held(lambda: block(*small, keep=True))[1]


def test_nothing_is_kept_without_a_gradient(block):
    leaves, _ = _leaves()
    with torch.no_grad():
        assert _held(lambda: block(*leaves, keep=True))[1] < 1 << 20
    assert _held(lambda: block(*(v.detach() for v in leaves), keep=True))[1] < 1 << 20


def test_no_room_for_it(block):
    """Memory that holds the call but not what it would keep: made again where the caller left the choice, an error where not."""
    from paper_2511_13645_amd import binding as fsa
    leaves, gy = _leaves()
    y = block(*leaves, keep=False)
    want = [y.detach().clone(), *torch.autograd.grad(y, leaves, gy)]
    del y
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    room = fsa.fsa_gated_fwd_workspace_bytes(T, D, H, O, torch.bfloat16) + (32 << 20)
    assert room + (32 << 20) < fsa.lib().fsa_gated_kept_bytes(T, D, H, O, 1)
    total = torch.cuda.mem_get_info()[1]
    try:
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + room) / total)
        with pytest.raises(torch.cuda.OutOfMemoryError):
            block(*leaves, keep=True)
        y = block(*leaves)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert torch.equal(y.detach(), want[0])
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, leaves, gy), want[1:]))

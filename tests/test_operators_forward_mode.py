"""Dual tensors of forward mode are refused by every operator, with gradients recorded or not: their tangents would be lost.  On the CPU, which comes before any look at the device."""
import pytest

torch = pytest.importorskip("torch")

from torch.autograd import forward_ad  # noqa: E402

from paper_1807_05358_amd import operators as O  # noqa: E402

H = torch.bfloat16


def calls(dual):
    """each operator with one of its tensors made dual"""
    x, m, w, h, n, u = torch.ones(3, 8), torch.ones(3, 8, dtype=H), torch.ones(8), torch.ones(2, 2, 1, 64, dtype=H), torch.ones(2, dtype=torch.int32), torch.ones(3)
    pages, table, targets = torch.ones(4, 2, 16, 64, dtype=H), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    yield lambda: O.layernorm_fwd(dual(x), w)
    yield lambda: O.layernorm_fwd(x, w, residual=dual(x))
    yield lambda: O.layernorm_bwd(x, x, dual(w), u, u)
    yield lambda: O.attention_fwd(h, dual(h), h)
    yield lambda: O.attention_bwd(dual(h), h, h, h, h, u)
    yield lambda: O.vocab_loss_fwd(m, dual(m), targets)
    yield lambda: O.vocab_loss_bwd(dual(u), m, m, targets, u)
    yield lambda: O.cache_write(h, dual(h), pages, pages, table, n)
    yield lambda: O.cache_write(h, h, dual(pages), pages, table, n)
    yield lambda: O.cache_read(pages, dual(pages), table, n)
    yield lambda: O.attention_paged_fwd(dual(h), pages, pages, table, n)
    yield lambda: O.sample(dual(x), u)


def test_tangents_are_not_lost():
    with forward_ad.dual_level():
        for call in calls(lambda t: forward_ad.make_dual(t, torch.ones_like(t))):
            for recorded in (True, False):
                with pytest.raises(ValueError, match="tangent"), torch.set_grad_enabled(recorded):
                    call()
        # tensors without a tangent come as far as outside
        for call in calls(lambda t: t):
            with pytest.raises(ValueError, match="no CPU path"):
                call()
    for call in calls(lambda t: t):
        with pytest.raises(ValueError, match="no CPU path"):
            call()


def test_under_jvp():
    for call in (lambda t: O.layernorm_fwd(t, torch.ones(8))[0], lambda t: O.sample(t, torch.ones(3))[1]):
        with pytest.raises(ValueError, match="tangent"):
            torch.func.jvp(call, (torch.ones(3, 8),), (torch.ones(3, 8),))

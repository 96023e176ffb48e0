"""Tensors that require gradients: autograd does not see the operators, so that they are refused where it would lose the gradients."""
import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import operators as O  # noqa: E402

BF16, F16 = torch.bfloat16, torch.float16


def calls():
    x, w = torch.zeros(4, 64, dtype=BF16), torch.zeros(64, dtype=BF16)
    f, t = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    q, lse = torch.zeros(2, 4, 8, 64, dtype=F16), torch.zeros(2, 4, 8)
    return [(O.layernorm_fwd, (x, w, w), dict(residual=x)), (O.layernorm_bwd, (x, x, w, f, f), dict(dh=x)), (O.attention_fwd, (q, q, q), {}),
            (O.attention_bwd, (q, q, q, q, q, lse), {}), (O.vocab_loss_fwd, (x, x, t), {}), (O.vocab_loss_bwd, (f, x, x, t, f), {})]


@pytest.mark.parametrize("n", range(6))
def test_tensors_that_require_gradients_are_refused(n):
    function, args, more = calls()[n]
    # without gradients the refusal is that of tensors in host memory, which comes after
    with pytest.raises(ValueError, match="no CPU path"):
        function(*args, **more)
    for name in [i for i, a in enumerate(args) if a.is_floating_point()] + list(more):
        a, m = [x.clone() for x in args], {k: x.clone() for k, x in more.items()}
        (a[name] if isinstance(name, int) else m[name]).requires_grad_()
        with pytest.raises(ValueError, match="requires gradients"):
            function(*a, **m)
        with torch.no_grad(), pytest.raises(ValueError, match="no CPU path"):
            function(*a, **m)

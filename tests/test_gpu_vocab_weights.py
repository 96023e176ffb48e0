"""The loss over a vocabulary where rows weigh very differently."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("top", [2.0 ** 14, 2.0 ** -3])
@pytest.mark.parametrize("rows,vocab,dim", [(200, 12, 64), (70, 3, 40), (500, 40, 520)])
def test_vocab_loss_weights_far_apart(rows, vocab, dim, top, dtype):
    """weights over 36 powers of two: in float16 g has steps of 2^-39 of the largest, so that dx of every row is as good as that allows"""
    from paper_1807_05358_amd import operators as ops
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + vocab)
    x = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") / math.sqrt(dim)).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    dloss = top * 2.0 ** (-36 * torch.rand(rows, generator=g, device="cuda"))
    dloss[rows // 2] = top
    lse = ops.vocab_loss_fwd(x, w, t)[1]
    dx, dw = ops.vocab_loss_bwd(dloss, x, w, t, lse)
    want = R.vocab_loss_bwd(dloss, x, w, t, lse)
    value, bound = want["dx"]
    if dtype == F16:        # the reference's steps are 2^-36 of the largest
        fewer = (2.0 ** -37 - 2.0 ** -40) * dloss.max().double()
        bound = bound - 1.01 * fewer * w.double().abs().sum(0)
    R.close(dx, value, bound, "dx")
    R.close(dw, *want["dw"], "dw")

"""The gradient of rows whose target has nearly all of the probability: its entry is p - 1, a difference."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,vocab,dim", [(64, 70, 64), (40, 1, 8), (500, 2000, 128), (1100, 12000, 520)])
def test_vocab_loss_of_confident_rows(rows, vocab, dim, dtype):
    """logits near 0 for the target and 4 to 16 below for the others, so that the statistics are near 0, too, and exact"""
    from paper_1807_05358_amd import operators as ops
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + vocab)
    x, w = torch.randn(rows, dim, generator=g, device="cuda") * 0.1, torch.randn(vocab, dim, generator=g, device="cuda") * 0.1
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    t[:] = t[0]                         # one word for all, which is the only one not far below
    far = torch.rand(rows, generator=g, device="cuda") * 12 + 4 + math.log(vocab)
    x[:, 0], w[:, 0] = -far, 1.0
    w[t[0].long(), 0] = 0.0
    x, w = x.to(dtype), w.to(dtype)
    _, lse, _ = ops.vocab_loss_fwd(x, w, t)
    dloss = torch.rand(rows, generator=g, device="cuda") + 0.5
    want = R.vocab_loss_bwd(dloss, x, w, t, lse)
    for name, got in zip(("dx", "dw"), ops.vocab_loss_bwd(dloss, x, w, t, lse)):
        R.close(got, *want[name], name)

"""The loss over a vocabulary where its products are large enough for tiles of 256 x 256 (tests/test_vocab_tiling.py holds that they are)."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402
from vocab_tile_cases import CASES  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_1807_05358_amd import operators
    return operators


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("what", list(CASES))
def test_vocab_loss_of_large_tiles(ops, what, dtype):
    rows, vocab, dim, ignored = CASES[what]
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + vocab + dim)
    x = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    w = (torch.randn(vocab, dim, generator=g, device="cuda") * (2 / math.sqrt(dim))).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    t[:4] = torch.tensor([0, vocab - 1, 255, vocab // 256 * 256], device="cuda")      # words at the edges of tiles
    t[torch.rand(rows, generator=g, device="cuda") < ignored] = -100
    got = ops.vocab_loss_fwd(x, w, t)
    for (name, (value, bound)), y in zip(R.vocab_loss_fwd(x, w, t).items(), got):
        R.close(y, value, bound, name)
    dloss = torch.rand(rows, generator=g, device="cuda") / rows
    first = ops.vocab_loss_bwd(dloss, x, w, t, got[1])
    want = R.vocab_loss_bwd(dloss, x, w, t, got[1])
    for name, y in zip(("dx", "dw"), first):
        R.close(y, *want[name], name)
    assert not first[0][t == -100].any()
    for a, b in zip(first, ops.vocab_loss_bwd(dloss, x, w, t, got[1])):
        assert torch.equal(a, b)

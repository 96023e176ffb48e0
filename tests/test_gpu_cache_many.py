"""A paged cache of more sequences times heads than a launch takes along a side, written, read back and attended over."""
import pytest

torch = pytest.importorskip("torch")

import answering_reference as R  # noqa: E402
from paper_1807_05358_amd import operators as O  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,K", [(40000, 2), (32767, 2), (32768, 2), (700, 200), (65535, 3)])
def test_read_back_what_was_written(B, K):
    P, D, t = 16, 8, torch.bfloat16
    torch.manual_seed(B)
    pages, n = B + 5, 7
    k_pages, v_pages = (torch.randn(pages, K, P, D, device="cuda").to(t) for _ in range(2))
    wide = torch.randperm(pages, device="cuda")[:B].int()[:, None].expand(B, 2).contiguous()
    wide[:, 1] = -1                                 # a second page that nobody has
    start = torch.randint(0, 9, (B,), device="cuda", dtype=torch.int32)
    k, v = (torch.randn(B, K, n, D, device="cuda").to(t) for _ in range(2))
    O.cache_write(k, v, k_pages, v_pages, wide, start)
    lengths = start + n
    lengths[::5] = 0
    got = O.cache_read(k_pages, v_pages, wide, lengths, kv_len=17)
    at = torch.arange(17, device="cuda")
    for g, x, p in zip(got, (k, v), (k_pages, v_pages)):
        assert g.shape == (B, K, 17, D)
        want = torch.where((at[:16] < lengths[:, None])[:, None, :, None], p[wide[:, 0].long()], 0)
        assert torch.equal(g[:, :, :16], want) and int(g[:, :, 16].count_nonzero()) == 0
        full = start.long()[:, None, None, None] + torch.arange(n, device="cuda")[None, None, :, None]
        assert torch.equal(p[wide[:, 0].long()].gather(2, full.expand(B, K, n, D)), x)
    some = torch.tensor([0, 1, B // 2, B - 2, B - 1], device="cuda")
    q = torch.randn(B, K, 1, D, device="cuda").to(t)
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, wide, lengths)
    want = R.attention(q[some], got[0][some].double(), got[1][some].double(), lengths[some])
    assert bool(((o[some].double() - want[0]).abs() <= want[1]).all())
    live = want[2].isfinite()
    assert torch.equal(lse[some].isfinite(), live) and bool(((lse[some].double() - want[2]).abs()[live] <= want[3][live]).all())


def test_no_sequences():
    pages, none = torch.zeros(3, 2, 16, 64, device="cuda").half(), torch.zeros(0, dtype=torch.int32, device="cuda")
    k, v = O.cache_read(pages, pages, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), none)
    assert k.shape == v.shape == (0, 2, 64, 64)

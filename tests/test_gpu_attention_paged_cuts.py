"""Attention over a paged cache at the limits of the rule that says whether sequences are cut into runs: 1023 blocks and 1024, tables of 2048 positions and more, of 1024 and more."""
import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import operators as O  # noqa: E402
from test_gpu_attention_paged import compare, filled  # noqa: E402

pytestmark = pytest.mark.gpu


def workspace(B, K, H, entries, P, D):
    """bytes of a call's workspace: none where no sequence is cut"""
    h, cache = O.ff_heads_t(1 << 20, 0, 0, 0), O.ff_cache_t(1 << 20, 1 << 20, 0, 0, 1 << 20, 0, 0, 0, 0, entries, 1, P, entries, O.FF_HELD_SAME)
    return O.workspace_bytes("ff_op_attention_paged_fwd", O.ff_attention_paged_fwd_t(O.FF_BF16, B, H, K, 1, D, 0, 1.0, h, h, cache, None, None, None, None, 0))


@pytest.mark.parametrize("B,K,entries,cut", [(1023, 1, 129, True), (1024, 1, 129, False), (1023, 1, 128, False), (511, 2, 129, True), (512, 2, 129, False), (511, 1, 65, True), (511, 1, 64, False), (512, 1, 65, False),
                                             (1, 1023, 129, True), (1, 1024, 129, False), (3, 341, 129, True)])
@pytest.mark.parametrize("held", ["same", "e4m3"])
def test_on_both_sides(B, K, entries, cut, held):
    """most sequences of a few positions or none, one as long as the table"""
    P = D = 16
    assert (workspace(B, K, 2 * K, entries, P, D) > 0) == cut
    lengths = [(i * 5) % 19 for i in range(B)]
    lengths[B // 2] = 16 * entries - 3
    # (compare() makes keys and values dense for all sequences: the long one would be of many)
    cache = filled([min(n, 40) for n in lengths], K, P, D, held, torch.bfloat16, more_entries=entries - 3)
    k_pages, v_pages, scales, tab, nk = cache
    q = torch.randn(B, 2 * K, 1, D, device="cuda").bfloat16()
    o, lse = compare(q, *cache)
    # the long sequence goes round the pages that it has
    b, mine = B // 2, tab[B // 2, :3].clone()
    tab[b] = mine[torch.arange(entries, device="cuda") % 2]
    nk[b] = lengths[b]
    x, y = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk, **scales)
    compare(q[b:b + 1], k_pages, v_pages, scales, tab[b:b + 1], nk[b:b + 1])
    one, two = O.attention_paged_fwd(q[b:b + 1], k_pages, v_pages, tab[b:b + 1], nk[b:b + 1], **scales)
    # cut elsewhere, or not: parts are rounded to 32 bits and joined, and an output may then round the other way, half a step each
    top = float(o.double().abs().max())
    assert float((x[b].double() - one[0].double()).abs().max()) <= 2.0 ** -8 * 2 * max(top, float(one.double().abs().max())) and float((y[b] - two[0]).abs().max()) <= 1e-5
    # the others do not depend on where they are cut, but by such roundings
    rest = torch.arange(B, device="cuda") != b
    assert torch.equal(lse[rest].isfinite(), y[rest].isfinite())
    assert float((lse[rest] - y[rest]).nan_to_num(0).abs().max() if B > 1 else 0) <= 1e-5 and float((o[rest].double() - x[rest].double()).abs().max() if B > 1 else 0) <= 2.0 ** -8 * 2 * top

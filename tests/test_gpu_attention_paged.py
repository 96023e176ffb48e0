"""Attention over a paged cache against its definition in 64 bits: types, ways to hold elements, head layouts, lengths, pages, masks that leave nothing, runs that cut sequences."""
import math

import pytest

torch = pytest.importorskip("torch")

import answering_reference as R  # noqa: E402
from operators_reference import close  # noqa: E402
from paper_1807_05358_amd import operators as O  # noqa: E402
from test_gpu_cache import TYPES, empty_cache, tables  # noqa: E402

pytestmark = pytest.mark.gpu
CUT = 1040         # positions more in the table: sequences are then cut into runs


def filled(lengths, K, P, D, held, t, seed=0, more_entries=0, spread=1.0):
    """(k_pages, v_pages, scales, table) with random values at all positions; behind them, and in pages that no sequence has, NaN; entries beyond the lengths are -1"""
    torch.manual_seed(seed)
    B, n = len(lengths), max(1, max(lengths))
    entries = -(-n // P) + more_entries
    pages = B * entries + 2
    k_pages, v_pages, scales = empty_cache(pages, K, P, D, held, t, fill=0xff)
    tab = tables(B, entries, pages, seed)
    nk = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    k, v = ((torch.randn(B, n, K, D, device="cuda") * spread).to(t).transpose(1, 2) for _ in range(2))
    O.cache_write(k, v, k_pages, v_pages, tab, torch.zeros_like(nk), lengths=nk, **scales)
    for b, m in enumerate(lengths):
        tab[b, -(-m // P):] = -1
    return k_pages, v_pages, scales, tab, nk


def compare(q, k_pages, v_pages, scales, tab, nk, **more):
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk, **more, **scales)
    S = max(1, int(nk.max()))
    k, v = (R.dense(p, scales.get(s), tab, nk.clamp(min=0), S, q.dtype) for p, s in ((k_pages, "k_scales"), (v_pages, "v_scales")))
    want = R.attention(q, k, v, nk, **more)
    assert o.shape == q.shape and o.dtype == q.dtype and lse.dtype == torch.float32
    close(lse, want[2], want[3], "lse")
    close(o, want[0], want[1], "o")
    return o, lse


CASES = [  # held, type, lengths, heads, kv_heads, queries, dim, page, causal
    ("same", "bf16", [1], 1, 1, 1, 64, 16, False),
    ("same", "f16", [5, 0, 17], 4, 2, 1, 128, 16, False),
    ("same", "bf16", [33, 16, 15], 8, 1, 1, 72, 32, False),
    ("same", "f16", [100, 64, 31], 12, 4, 2, 8, 16, True),
    ("same", "bf16", [700, 3, 257, 512], 8, 8, 1, 128, 16, False),
    ("same", "f16", [1, 2000, 0, 0, 900, 13], 6, 2, 3, 64, 64, True),
    ("same", "bf16", [300, 1], 48, 2, 1, 96, 16, False),                      # 24 columns
    ("same", "bf16", [90, 40], 32, 4, 9, 128, 128, True),                     # 72 columns, three blocks of them
    ("e4m3", "bf16", [1, 40], 4, 4, 1, 128, 16, False),
    ("e4m3", "f16", [333, 0, 800], 8, 2, 1, 80, 32, False),
    ("e4m3", "bf16", [65, 130], 2, 2, 5, 16, 16, True),
    ("e4m3", "f16", [1500, 600], 20, 1, 1, 64, 256, False),
    ("e2m1", "bf16", [31, 2], 4, 2, 1, 64, 16, False),
    ("e2m1", "f16", [900, 0, 77, 260], 8, 8, 2, 128, 32, True),
    ("e2m1", "bf16", [410], 16, 2, 4, 96, 64, True),
    ("e2m1", "f16", [50, 49, 48], 3, 3, 1, 32, 16, False),
]


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("held,t,lengths,H,K,n,D,P,causal", CASES)
def test_against_the_definition(held, t, lengths, H, K, n, D, P, causal, cut):
    """by a block for each sequence, and, with a table for long ones, by runs of tiles"""
    t = TYPES[t]
    cache = filled(lengths, K, P, D, held, t, seed=D + n, more_entries=CUT // P if cut else 0)
    q = (1.5 * torch.randn(len(lengths), n, H, D, device="cuda")).to(t).transpose(1, 2)
    o, _ = compare(q, *cache, causal=causal)
    assert o.stride() == q.stride()                                           # an output in the queries' order
    again, _ = O.attention_paged_fwd(q, cache[0], cache[1], cache[3], cache[4], causal=causal, **cache[2])
    assert torch.equal(o, again)


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
def test_lengths_of_queries_and_masks_that_leave_nothing(held, cut):
    lengths = [3, 40, 0, 600, 7]
    cache = filled(lengths, 2, 16, 64, held, torch.bfloat16, more_entries=CUT // 16 if cut else 0)
    q = torch.randn(5, 4, 6, 64, device="cuda").bfloat16()
    for q_lengths in ([6, 2, 3, 0, -1], [1, 6, 6, 9, 5]):
        nq = torch.tensor(q_lengths, dtype=torch.int32, device="cuda")
        q[3, :, 1] = math.nan                     # a query that takes no part, or one that does
        for causal in (False, True):
            qq = q.clone()
            if q_lengths[3]:
                qq[3, :, 1] = 0.5
            compare(qq, *cache, causal=causal, q_lengths=nq)


def test_lengths_outside_the_table_are_clamped():
    k_pages, v_pages, scales, tab, nk = filled([64, 32], 1, 16, 64, "same", torch.float16)
    tab[1] = tab[0]
    q = torch.randn(2, 2, 1, 64, device="cuda").half()
    a = O.attention_paged_fwd(q, k_pages, v_pages, tab, torch.tensor([2 ** 31 - 1, -7], dtype=torch.int32, device="cuda"))
    b = O.attention_paged_fwd(q, k_pages, v_pages, tab, torch.tensor([64, 0], dtype=torch.int32, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and int(a[0][1].count_nonzero()) == 0 and bool((a[1][1] == -math.inf).all())


@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
@pytest.mark.parametrize("lengths,cut", [([40, 100], False), ([900, 600], False), ([40, 100], True), ([900, 600], True)])
def test_a_missing_page_is_loud(held, lengths, cut):
    """queries that see the positions of an entry that is no page get NaN, the others their values"""
    for entry in (-1, 10 ** 6):
        cache = filled(lengths, 2, 16, 64, held, torch.bfloat16, more_entries=CUT // 16 if cut else 0)
        cache[3][0, 1] = entry                    # positions 16 .. 31 of the first sequence
        q = torch.randn(2, 4, 1, 64, device="cuda").bfloat16()
        o, lse = compare(q, *cache)
        assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(lse[0]).all()) and bool(torch.isfinite(o[1]).all())
    # causal: the first queries of many see only what lies before it
    cache = filled([40], 2, 16, 64, held, torch.bfloat16)
    cache[0].view(torch.uint8)[0] = 0             # the page that is looked at instead is not to make a NaN of them
    cache[1].view(torch.uint8)[0] = 0
    for s in cache[2].values():
        s[0] = 0
    cache[3][0, 2] = -1
    q = torch.randn(1, 2, 20, 64, device="cuda").bfloat16()
    o, lse = O.attention_paged_fwd(q, cache[0], cache[1], cache[3], cache[4], causal=True, **cache[2])
    bad = torch.isnan(lse[0, 0])
    assert bad.tolist() == [False] * 12 + [True] * 8 and bool(torch.isfinite(o[0, :, :12]).all()) and bool(torch.isnan(o[0, :, 12:]).all())


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
def test_a_missing_page_leaves_the_others_alone(t, held, cut):
    """whatever lies in the page that is read in its place: queries that do not see the missing positions keep their values"""
    for n, lengths in ((20, [40]), (3, [1200])):
        k_pages, v_pages, scales, tab, nk = filled(lengths, 2, 16, 64, held, t, more_entries=CUT // 16 if cut else 0)
        free = next(i for i in range(len(k_pages)) if i and i not in tab.tolist()[0])
        for x in (k_pages.view(torch.uint8), v_pages.view(torch.uint8), *scales.values()):
            x[free] = x[0]
            x[0] = 0xff                           # NaN, of elements and of scales
        tab[tab == 0] = free
        last = -(-lengths[0] // 16) - 1
        q = torch.randn(1, 2, n, 64, device="cuda").to(t)
        whole = [x.clone() for x in compare(q, k_pages, v_pages, scales, tab, nk, causal=True)]
        tab[0, last] = -1
        o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk, causal=True, **scales)
        sees = [i + lengths[0] - n >= 16 * last for i in range(n)]
        assert torch.isnan(lse[0, 0]).tolist() == sees and torch.isnan(o[0]).all(2)[1].tolist() == sees
        for x, y in zip((o, lse), whole):
            assert torch.equal(x[0][:, :n - sum(sees)], y[0][:, :n - sum(sees)])
        # queries that are padding see none of it
        o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk, q_lengths=torch.ones_like(nk), **scales)
        assert bool(torch.isnan(o[0, :, 0]).all()) and int(o[0, :, 1:].count_nonzero()) == 0 and bool((lse[0, :, 1:] == -math.inf).all())


@pytest.mark.parametrize("cut", [False, True])
def test_padding_beside_values_that_are_not_finite(cut):
    k_pages, v_pages, scales, tab, nk = filled([1100, 30], 1, 16, 64, "same", torch.bfloat16, more_entries=CUT // 16 if cut else 0)
    v_pages[tab[:, 0].long(), 0, 3, 7] = math.inf
    q = torch.randn(2, 2, 3, 64, device="cuda").bfloat16()
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk, q_lengths=torch.tensor([2, 0], dtype=torch.int32, device="cuda"))
    assert bool(torch.isinf(o[0, :, :2, 7]).all()) and int((~torch.isfinite(o)).sum()) == 4
    assert int(o[0, :, 2].count_nonzero()) == int(o[1].count_nonzero()) == 0 and bool((lse[0, :, 2] == -math.inf).all()) and bool((lse[1] == -math.inf).all())


def test_large_scores_and_values():
    """scores far apart, where all but a few keys weigh nothing; rows of values at the type's ends"""
    for t in (torch.float16, torch.bfloat16):
        cache = filled([500, 64], 2, 16, 128, "same", t, spread=6.0, more_entries=CUT // 16)
        q = (6 * torch.randn(2, 4, 1, 128, device="cuda")).to(t)
        compare(q, *cache)
        compare(q, *cache, scale=2.0)
        cache[1].nan_to_num_(0.0).clamp_(-1, 1).mul_(30000.0 if t == torch.float16 else 2.0 ** 120)
        compare(q, *cache)


def test_many_keys_that_weigh_little_beside_one_without_a_value():
    """4096 keys 14 below one key: in float16 their probabilities are kept times 2^8"""
    for t in (torch.float16, torch.bfloat16):
        k_pages, v_pages, scales, tab, nk = filled([4097], 1, 16, 64, "same", t)
        k_pages.zero_(), v_pages.fill_(1.0)
        k_pages[tab[0, 0].long(), 0, 0, 0], v_pages[tab[0, 0].long(), 0, 0] = 14.0, 0.0
        q = torch.zeros(1, 1, 1, 64, device="cuda", dtype=t)
        q[..., 0] = 1
        compare(q, k_pages, v_pages, scales, tab, nk, scale=1.0)


def test_infinities_and_nans_reach_the_queries_that_see_them():
    k_pages, v_pages, scales, tab, nk = filled([50, 50], 1, 16, 64, "same", torch.bfloat16)
    k_pages[tab[0, 2].long(), 0, 1, 5] = math.nan                               # position 33 of the first sequence
    v_pages[tab[1, 0].long(), 0, 3, 7] = math.inf
    q = torch.randn(2, 2, 1, 64, device="cuda").bfloat16()
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk)
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(lse[0]).all())
    assert bool(torch.isinf(o[1, :, 0, 7]).all()) and int((~torch.isfinite(o[1])).sum()) == 2 and bool(torch.isfinite(lse[1]).all())
    # beyond a length they are not read
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, torch.tensor([33, 3], dtype=torch.int32, device="cuda"))
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())


def test_many_sequences():
    """more sequences than threads of a block, most of them short or empty, one long"""
    lengths = [(i * 7) % 23 if i % 3 else 0 for i in range(700)]
    lengths[350] = 2600
    for held in ("same", "e4m3"):
        cache = filled(lengths, 1, 16, 64, held, torch.bfloat16)
        q = torch.randn(700, 2, 1, 64, device="cuda").bfloat16()
        compare(q, *cache)
    # and so many blocks that no sequence is cut
    lengths = [600, 0, 300] + [20] * 253
    cache = filled(lengths, 16, 16, 32, "same", torch.float16)
    q = torch.randn(256, 16, 1, 32, device="cuda").half()
    compare(q, *cache)


def test_one_sequence_in_many_runs():
    cache = filled([20000, 30], 1, 16, 64, "e4m3", torch.bfloat16, more_entries=100)
    compare(torch.randn(2, 5, 1, 64, device="cuda").bfloat16(), *cache)


def test_shared_pages_and_strided_queries():
    """two sequences with the same beginning; queries that are copied because their rows do not begin at multiples of 16 bytes; a wider table"""
    k_pages, v_pages, scales, tab, nk = filled([48, 48], 2, 16, 64, "e2m1", torch.float16)
    tab = torch.cat([tab, tab], 1)[:, :3]
    tab[1, :2] = tab[0, :2]
    q = torch.randn(2, 6, 2, 67, device="cuda").half()[..., 1:65]
    compare(q, k_pages, v_pages, scales, tab, nk, causal=True)
    compare(q.transpose(1, 2).contiguous().transpose(1, 2), k_pages, v_pages, scales, tab, nk, causal=True)


def test_like_the_contiguous_kernel():
    """the same keys in pages and dense: outputs alike but for roundings"""
    cache = filled([513, 100], 4, 64, 128, "same", torch.bfloat16)
    k, v = O.cache_read(*cache[:2], cache[3], cache[4], kv_len=513)
    q = torch.randn(2, 8, 1, 128, device="cuda").bfloat16()
    a, b = O.attention_paged_fwd(q, *cache[:2], cache[3], cache[4]), O.attention_fwd(q, k, v, kv_lengths=cache[4])
    # two roundings to bfloat16 of an output below 1, and that of the probabilities in one of them
    assert float((a[0].double() - b[0].double()).abs().max()) <= 3 * 2.0 ** -8 * float(b[0].double().abs().max()) and float((a[1] - b[1]).abs().max()) < 1e-5


def test_captured_and_replayed():
    """a step in a graph, replayed with other lengths and queries, eager work between; a second graph of the same cache beside it"""
    cache = filled([900, 300], 2, 16, 64, "same", torch.bfloat16, more_entries=CUT // 16)
    k_pages, v_pages, scales, tab, nk = cache
    q = torch.randn(2, 4, 1, 64, device="cuda").bfloat16()
    new = torch.randn(2, 2, 1, 64, device="cuda").bfloat16()
    start = nk - 1

    def step():
        O.cache_write(new, new, k_pages, v_pages, tab, start)
        return O.attention_paged_fwd(q, k_pages, v_pages, tab, nk)

    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for n in (900, 899, 17, 1, 640):
        nk[0] = n
        start.copy_(nk - 1)
        q.copy_(torch.randn_like(q)), new.copy_(torch.randn_like(new))
        for g, _ in graphs:
            g.replay()
        results = [[x.clone() for x in out] for _, out in graphs]
        want = step()
        torch.cuda.synchronize()
        for r in results:
            assert all(torch.equal(x, y) for x, y in zip(r, want))


def test_on_two_streams_at_once():
    """each call has a workspace of its own"""
    cache = filled([5000, 300], 2, 16, 64, "e4m3", torch.bfloat16)
    qs = [torch.randn(2, 4, 1, 64, device="cuda").bfloat16() for _ in range(2)]

    def call(q):
        return O.attention_paged_fwd(q, cache[0], cache[1], cache[3], cache[4], **cache[2])

    want = [call(q) for q in qs]
    got = []
    for q in qs:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([call(q) for _ in range(10)])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, several in zip(want, got) for g in several for x, y in zip(g, w))


def test_as_many_sequences_and_queries_as_there_may_be():
    """65535 sequences, cut and not, each as it is by itself; one head's 65535 * 16 queries"""
    B, D, t = 65535, 8, torch.bfloat16
    k_pages, v_pages = (torch.randn(64, 1, 16, D, device="cuda").to(t) for _ in range(2))
    some = torch.tensor([0, 1, 255, 256, 32768, B - 1], device="cuda")
    for entries in (2, 70):
        tab = torch.randint(0, 64, (B, entries), dtype=torch.int32, device="cuda")
        nk = torch.randint(0, 33, (B,), dtype=torch.int32, device="cuda")
        q = torch.randn(B, 1, 1, D, device="cuda").to(t)
        o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk)
        a, b = O.attention_paged_fwd(q[some], k_pages, v_pages, tab[some], nk[some])
        c, d = compare(q[some], k_pages, v_pages, {}, tab[some], nk[some])
        # parts of a sequence are joined where another call does not cut it: a rounding to float32 each, and one to the type that may fall the other way
        assert float((lse[some] - d).nan_to_num(0).abs().max()) < 1e-5 and float((o[some].float() - c.float()).abs().max()) <= 2.0 ** -8 * float(v_pages.float().abs().max())
        assert torch.equal(a, c) and torch.equal(b, d)
    n = 65535 * 16
    q = torch.randn(1, 1, n, D, device="cuda").to(t)
    tab, nk = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([41], dtype=torch.int32, device="cuda")
    o, lse = O.attention_paged_fwd(q, k_pages, v_pages, tab, nk)
    for at in (0, n // 2 + 5, n - 3):
        x, y = compare(q[:, :, at:at + 3].contiguous(), k_pages, v_pages, {}, tab, nk)
        assert torch.equal(x, o[:, :, at:at + 3]) and torch.equal(y, lse[:, :, at:at + 3])

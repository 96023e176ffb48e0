"""CPU-side checks of the operators that a decoder answers with: malformed records are refused before anything is launched, the functions refuse what they cannot take, and the arithmetic
that deals tiles of the paged attention and looks up pages stays within what there is, on the host."""
import ctypes as C
import os
import random
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import binding, operators as O  # noqa: E402
from test_operators_refusals import P, code, put  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_05358_amd", "csrc", "ffops_paged_runs.h")
INVALID, RANGE, WORKSPACE = binding.FF_EINVAL, binding.FF_ERANGE, binding.FF_EWORKSPACE
NAN, INF = float("nan"), float("inf")


def good(name):
    h = O.ff_heads_t(P, 8 * 16 * 64, 16 * 64, 64)
    cache = O.ff_cache_t(P, P, P, P, P, 4096, 4096, 64, 64, 8, 4, 16, 8, O.FF_HELD_SAME)
    if name == "ff_op_cache_write":
        return O.ff_cache_write_t(O.FF_BF16, 2, 2, 64, 3, h, h, cache, P, P)
    if name == "ff_op_cache_read":
        return O.ff_cache_read_t(O.FF_BF16, 2, 2, 64, 3, h, h, cache, P)
    if name == "ff_op_attention_paged_fwd":
        return O.ff_attention_paged_fwd_t(O.FF_BF16, 2, 8, 2, 1, 64, 0, 0.125, h, h, cache, P, P, P, P, 1 << 30)
    return O.ff_sample_t(O.FF_F32, 2, 100, O.ff_rows_t(P, 100), P, None, None, None, None, 1.0, 1.0, 0.0, 0, P, P)


CACHE = [(INVALID, dict(dtype=O.FF_F32)), (INVALID, dict(dtype=9)), (INVALID, dict(kv_heads=0)), (INVALID, dict(head_dim=0)), (INVALID, dict(head_dim=60)), (RANGE, dict(head_dim=136)),
         (INVALID, dict(cache__held=3)), (INVALID, dict(cache__held=1, head_dim=72)), (INVALID, dict(cache__held=2, head_dim=80)), (INVALID, dict(cache__page=8)), (INVALID, dict(cache__page=24)),
         (RANGE, dict(cache__page=65536)), (RANGE, dict(cache__table_pages=(1 << 24) + 1)), (INVALID, dict(cache__pages=1 << 31)), (RANGE, dict(batch=65536)), (INVALID, dict(cache__pages=0)),
         (INVALID, dict(cache__table=None)), (INVALID, dict(cache__k=None)), (INVALID, dict(cache__v=None)), (INVALID, dict(cache__k=P + 8)), (INVALID, dict(cache__v=P + 2)), (INVALID, dict(cache__k_stride=4100)),
         (INVALID, dict(cache__v_stride=8)), (INVALID, dict(cache__held=1, cache__k_scale=None)), (INVALID, dict(cache__held=1, cache__v_scale=None)), (INVALID, dict(cache__held=2, cache__k_scale=P + 2)),
         (INVALID, dict(cache__held=1, cache__v_scale_stride=66))]
BAD = {
    "ff_op_cache_write": CACHE + [(INVALID, dict(k__p=None)), (INVALID, dict(v__p=P + 8)), (INVALID, dict(k__pos=60)), (INVALID, dict(start=None)), (RANGE, dict(new_len=1 << 27)), (RANGE, dict(new_len=1 << 28, kv_heads=1))],
    "ff_op_cache_read": CACHE + [(INVALID, dict(k__p=None)), (INVALID, dict(v__head=4)), (RANGE, dict(kv_len=1 << 28)), (RANGE, dict(batch=40000))],
    "ff_op_attention_paged_fwd": CACHE + [(INVALID, dict(heads=0)), (INVALID, dict(heads=7)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=NAN)), (INVALID, dict(scale=INF)), (INVALID, dict(q__p=None)),
                                          (INVALID, dict(o__p=P + 4)), (INVALID, dict(q__pos=12)), (INVALID, dict(lse=None)), (RANGE, dict(heads=65536 * 2)), (RANGE, dict(q_len=65535 * 4 + 1)),
                                          (WORKSPACE, dict(cache__table_pages=1000, workspace=None)), (WORKSPACE, dict(cache__table_pages=1000, workspace_bytes=100)),
                                          (WORKSPACE, dict(cache__table_pages=1000, workspace=P + 16))],
    "ff_op_sample": [(INVALID, dict(dtype=3)), (INVALID, dict(vocab=0)), (RANGE, dict(vocab=(1 << 24) + 1)), (RANGE, dict(rows=1 << 22)), (INVALID, dict(logits__p=None)), (INVALID, dict(u=None)),
                     (INVALID, dict(words=None)), (INVALID, dict(logprob=None))],
}


@pytest.mark.parametrize("name", sorted(BAD))
def test_malformed_records_are_refused(name):
    assert getattr(O.lib(), name)(None, None) == INVALID
    for want, fields in BAD[name]:
        assert code(name, put(good(name), **fields)) == want, fields
    if name + "_workspace_bytes" in O.EXPORTS:
        size = getattr(O.lib(), name + "_workspace_bytes")
        assert size(None) == 0 and size(C.byref(put(good(name), dtype=9))) == 0


def test_nothing_to_do_is_fine():
    for name in ("ff_op_cache_write", "ff_op_cache_read", "ff_op_attention_paged_fwd"):
        assert code(name, put(good(name), batch=0)) == 0
    assert code("ff_op_cache_write", put(good("ff_op_cache_write"), new_len=0)) == 0
    assert code("ff_op_cache_write", put(good("ff_op_cache_write"), cache__table_pages=0)) == 0
    assert code("ff_op_cache_read", put(good("ff_op_cache_read"), kv_len=0)) == 0
    assert code("ff_op_attention_paged_fwd", put(good("ff_op_attention_paged_fwd"), q_len=0)) == 0
    assert code("ff_op_sample", put(good("ff_op_sample"), rows=0)) == 0


def test_workspace_stays_bounded():
    size = lambda **f: O.workspace_bytes("ff_op_attention_paged_fwd", put(good("ff_op_attention_paged_fwd"), **f))
    assert size() == 0                                              # 128 positions: a block takes a sequence
    assert size(cache__table_pages=1000) > 0
    for heads, kv_heads, q_len, batch in ((32, 8, 1, 8), (64, 1, 1000, 2), (16, 16, 4096, 1), (128, 128, 8, 3), (32, 8, 1, 65535)):
        # 1024 blocks of 32 columns, two parts each, rounded up to whole runs of a key head
        assert size(heads=heads, kv_heads=kv_heads, q_len=q_len, batch=batch, head_dim=128, cache__table_pages=1 << 20) <= 2 * 2048 * 32 * 129 * 4


def test_functions_refuse_what_they_cannot_take():
    h, f8, u8 = torch.bfloat16, torch.float8_e4m3fn, torch.uint8
    q, pages, tab, n = torch.zeros(2, 4, 1, 64, dtype=h), torch.zeros(5, 2, 16, 64, dtype=h), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    new, z, u = torch.zeros(2, 2, 3, 64, dtype=h), torch.zeros(3, 50), torch.zeros(3)
    for bad in (lambda: O.cache_write(new, new, pages, pages, tab, n), lambda: O.cache_read(pages, pages, tab, n), lambda: O.attention_paged_fwd(q, pages, pages, tab, n), lambda: O.sample(z, u),     # not on a GPU
                lambda: O.cache_write(new[0], new, pages, pages, tab, n), lambda: O.attention_paged_fwd(q[0], pages, pages, tab, n), lambda: O.sample(z[0], u),
                lambda: O.cache_write(new.float(), new.float(), pages, pages, tab, n), lambda: O.sample(z.double(), u), lambda: O.sample(z[:, :0], u)):
        with pytest.raises(ValueError):
            bad()
    # a cache that autograd would follow: writing and reading are not recorded
    leaf = pages.clone().requires_grad_()
    for call in (lambda: O.cache_write(new, new, leaf, pages, tab, n), lambda: O.cache_read(leaf, pages, tab, n), lambda: O.attention_paged_fwd(q, pages, leaf, tab, n)):
        with pytest.raises(ValueError, match="gradients"):
            call()
    # of a cache, as of one on a GPU
    meta = lambda *s, dtype: torch.empty(*s, dtype=dtype, device="meta")

    class Elsewhere:
        """a tensor's shape, type and strides, as of one on a GPU"""
        def __init__(self, t):
            self.t, self.is_cuda, self.device = t, True, "cuda:0"

        def __getattr__(self, name):
            return getattr(self.t, name)

        def data_ptr(self):
            return P

    def cache(pages, k_scales=None, v_scales=None, tab=tab, dtype=h, v=None):
        e = [None if x is None else Elsewhere(x) for x in (pages, pages if v is None else v, tab, k_scales, v_scales)]
        return O._cache_args(*e, dtype)

    K, D, values = cache(meta(5, 2, 16, 64, dtype=h))
    assert (K, D, values[5:9], values[10:]) == (2, 64, (2 * 16 * 64 * 2, 2 * 16 * 64 * 2, 0, 0), (5, 16, 3, O.FF_HELD_SAME))
    s1, s3 = meta(5, 2, 1, 16, dtype=u8), meta(5, 2, 3, 16, dtype=u8)
    assert cache(meta(5, 2, 16, 80, dtype=f8), s1, s1)[1] == 80 and cache(meta(5, 2, 16, 48, dtype=u8), s3, s3)[1] == 96
    room = meta(5, 3, 2, 16, 64, dtype=h)[:, 1]
    assert cache(room)[2][5] == 3 * 2 * 16 * 64 * 2
    for bad in (lambda: cache(meta(5, 2, 16, dtype=h)), lambda: cache(meta(5, 2, 16, 64, dtype=torch.float16)), lambda: cache(meta(5, 2, 16, 64, dtype=torch.float32)), lambda: cache(meta(5, 2, 24, 64, dtype=h)),
                lambda: cache(meta(5, 2, 8, 64, dtype=h)), lambda: cache(meta(5, 2, 65536, 64, dtype=h)), lambda: cache(meta(5, 2, 16, 136, dtype=h)), lambda: cache(meta(5, 2, 16, 60, dtype=h)), lambda: cache(meta(0, 2, 16, 64, dtype=h)),
                lambda: cache(meta(5, 16, 2, 64, dtype=h).transpose(1, 2)), lambda: cache(meta(5, 2, 16, 128, dtype=h)[..., :64]), lambda: cache(meta(5, 2, 16, 64, dtype=h), s1, s1),
                lambda: cache(meta(5, 2, 16, 64, dtype=f8)), lambda: cache(meta(5, 2, 16, 64, dtype=f8), s1), lambda: cache(meta(5, 2, 16, 64, dtype=f8), s3, s3), lambda: cache(meta(5, 2, 16, 72, dtype=f8), s1, s1),
                lambda: cache(meta(5, 2, 16, 40, dtype=u8), s3, s3), lambda: cache(meta(5, 2, 16, 64, dtype=h), tab=tab.long()), lambda: cache(meta(5, 2, 16, 64, dtype=h), tab=tab[0]),
                lambda: cache(meta(5, 2, 16, 64, dtype=h), v=meta(4, 2, 16, 64, dtype=h)), lambda: cache(meta(5, 2, 16, 64, dtype=h), tab=torch.zeros(3, 2, dtype=torch.int32).t())):
        with pytest.raises(ValueError):
            bad()


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(lines) -> numbers that the header's functions give"""
    at = tmp_path_factory.mktemp("runs")
    (at / "ask.cpp").write_text(f'''#include "{HEADER}"
#include <cstdio>
using namespace ffops;
int main()
{{
    char what;
    long long a, b, c;
    while (scanf(" %c %lld %lld %lld", &what, &a, &b, &c) == 4) {{
        if (what == 'u') printf("%u\\n", runs_used((uint32_t)a, b).n);
        else if (what == 'b') printf("%lld\\n", (long long)runs_used((uint32_t)b, c).begin((uint32_t)a));
        else if (what == 'o') printf("%u\\n", runs_used((uint32_t)b, c).of(a));
        else if (what == 'e') printf("%u\\n", entry_of((int)a, (int)b, (uint32_t)c));
        else if (what == 'p') printf("%u\\n", place_of((int)a, (int)b, (uint32_t)c));
        else printf("%u\\n", runs_of(a, b, c));
    }}
}}
''')
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-o", str(at / "ask"), str(at / "ask.cpp")])

    def run(lines):
        said = subprocess.run([str(at / "ask")], input="".join(f"{w} {x} {y} {z}\n" for w, x, y, z in lines), text=True, stdout=subprocess.PIPE, check=True).stdout
        return [int(x) for x in said.split()]
    return run


def test_runs_cover_every_tile_once(ask):
    """every tile is in one run, every run has one, run_of finds it; also where the list is far beyond 32 bits"""
    rng = random.Random(4)
    for _ in range(60):
        runs, all_ = rng.choice([1, 2, 7, 64, 1024]), rng.choice([1, 7, 8, 9, 100, 8191, rng.randint(1, 5000), (1 << 32) + 5, 65535 << 23])
        used = ask([("u", runs, all_, 0)])[0]
        assert 1 <= used <= runs and used <= max(1, -(-all_ // 8))
        begins = ask([("b", r, used, all_) for r in range(used + 1)])
        assert begins[0] == 0 and begins[-1] == all_ and all(x < y for x, y in zip(begins, begins[1:]))
        tiles = sorted({t for r in begins for t in (r - 1, r, r + 1) if 0 <= t < all_} | {rng.randrange(all_) for _ in range(20)})
        for t, r in zip(tiles, ask([("o", t, used, all_) for t in tiles])):
            assert begins[r] <= t < begins[r + 1]


def test_places_are_within_the_table_and_the_page(ask):
    for page in (16, 32, 256, 32768):
        for nk in (1, 15, 16, 17, 31, 32, 33, 255, 256, 257, 1 << 28):
            ats = [x for tile in {0, nk // 64, (nk - 1) // 32} for x in (tile * 32, tile * 32 + 16)]
            entries, places = ask([("e", x, nk, page.bit_length() - 1) for x in ats]), ask([("p", x, nk, page) for x in ats])
            for x, e, p in zip(ats, entries, places):
                assert 0 <= e <= (nk - 1) // page and 0 <= p <= page - 16 and p % 16 == 0
                if x < nk:
                    assert e * page + p == x


def test_sequences_are_cut_only_where_blocks_are_few(ask):
    assert ask([("r", 8, 8, 16384)]) == [64] and ask([("r", 1, 1, 1040)]) == [5] and ask([("r", 600, 1, 16384)]) == [1] and ask([("r", 16, 32, 4096)]) == [32]
    assert ask([("r", 8, 1, 1024), ("r", 64, 64, 16384), ("r", 5000, 1, 16384), ("r", 16, 32, 2048)]) == [0, 0, 0, 0]

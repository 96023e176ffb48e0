"""How the products of the vocabulary's loss are cut, on the host: the sizes that are tested for the large tiles take them, and no product is cut into what it does not have."""
import os
import random
import subprocess

import pytest

from vocab_tile_cases import CASES

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_05358_amd", "csrc", "ffops_vocab_tiling.h")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask([(m, n, k, split)]) -> [(tile, ms, ns, splits)], ask.pieces([(rows, vocab)]) -> [words]"""
    at = tmp_path_factory.mktemp("tiling")
    (at / "ask.cpp").write_text(f'''#include "{HEADER}"
#include <cstdio>
int main()
{{
    char what;
    unsigned long long m, n, k;
    int split;
    while (scanf(" %c %llu %llu %llu %d", &what, &m, &n, &k, &split) == 5) {{
        const ffops::Tiling t = ffops::tiling_of(m, n, k, split != 0);
        if (what == 't') printf("%u %u %u %u\\n", t.tile, t.ms, t.ns, t.splits);
        else printf("%u\\n", ffops::piece_of((uint32_t)m, (uint32_t)n));
    }}
}}
''')
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-o", str(at / "ask"), str(at / "ask.cpp")])

    def run(what, rows):
        said = subprocess.run([str(at / "ask")], input="".join(f"{what} {' '.join(map(str, r))}\n" for r in rows), text=True, stdout=subprocess.PIPE, check=True).stdout
        return [tuple(map(int, line.split())) for line in said.splitlines()]

    def tilings(products):
        return run("t", [(m, n, k, int(split)) for m, n, k, split in products])
    tilings.pieces = lambda sizes: [p for p, in run("p", [(r, v, 0, 0) for r, v in sizes])]
    return tilings


def test_cases_of_large_tiles_take_them(ask):
    seen = set()
    for what, (rows, vocab, dim, _) in CASES.items():
        d, piece = -(-dim // 8) * 8, ask.pieces([(rows, vocab)])[0]
        words, last = min(vocab, piece), (vocab - 1) % piece + 1
        fwd, z, zl, dx, dw, dwl = ask([(vocab, rows, d, False), (words, rows, d, False), (last, rows, d, False), (d, rows, words, True), (d, words, rows, True), (d, last, rows, True)])
        assert [t[0] for t in (fwd, z, zl, dx, dw, dwl)] == [256] * 6, what
        assert dim % 64 and rows % 256 and vocab % 256, what        # k, rows and words that end inside a tile
        pieces = vocab > piece
        seen |= {("dx", dx[3] > 1, pieces), ("dw", dwl[3] > 1)}
    # dx: at once, over splits, over pieces, over both; dw: at once, over splits
    assert seen == {("dx", False, False), ("dx", True, False), ("dx", False, True), ("dx", True, True), ("dw", False), ("dw", True)}


def test_any_product_is_covered_by_its_tiles(ask):
    rng = random.Random(5)
    products = [(int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(3, 17)), rng.random() < 0.5) for _ in range(2000)]
    for (m, n, k, split), (tile, ms, ns, splits) in zip(products, ask(products)):
        assert tile in (64, 128, 256) and ms == -(-m // tile) and ns == -(-n // tile)
        assert 1 <= splits <= 16 and (splits == 1 or split and k // splits >= 512)

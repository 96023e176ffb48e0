"""The bins of the choice of a word, on the host: between the logits that a bin's edges are taken for lie all words that are counted in it."""
import os
import random
import struct
import subprocess

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_05358_amd", "csrc", "ffops_sample_bins.h")


def single(x):
    return struct.unpack("f", struct.pack("f", x))[0]


def near(x, steps):
    """floats next to one another around x"""
    b = struct.unpack("i", struct.pack("f", x))[0]
    b = b if b >= 0 else -(b & 0x7fffffff)
    return [struct.unpack("f", struct.pack("I", n if n >= 0 else -n | 0x80000000))[0] for n in range(b - steps, b + steps + 1)]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask([(anchor, temperature, bins a unit, logit)]) -> [(the logit's bin, the logits on the safe side of its edges)]"""
    at = tmp_path_factory.mktemp("bins")
    (at / "ask.cpp").write_text(f'''#include "{HEADER}"
#include <cstdio>
int main()
{{
    float anchor, temperature, z;
    int per;
    while (scanf("%a %a %d %a", &anchor, &temperature, &per, &z) == 4) {{
        ffops::Bins b;
        b.set(anchor, temperature, per);
        const int n = b.bin(b.place(z));
        printf("%d %a %a\\n", n, b.logit(n, -1), b.logit(n + 1, 1));
    }}
}}
''')
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-o", str(at / "ask"), str(at / "ask.cpp")])

    def run(cases):
        said = subprocess.run([str(at / "ask")], input="".join(f"{a.hex()} {t.hex()} {p} {z.hex()}\n" for a, t, p, z in cases), text=True, stdout=subprocess.PIPE, check=True).stdout
        return [(int(n), float.fromhex(lo), float.fromhex(hi)) for n, lo, hi in (line.split() for line in said.splitlines())]
    return run


def hold(ask, cases):
    for (a, t, p, z), (n, lo, hi) in zip(cases, ask(cases)):
        if 0 <= n < 4096:
            assert lo <= z <= hi, (a, t, p, z, n, lo, hi)


def test_a_logit_of_0(ask):
    """which an edge may be next to, where nothing of it is left to be relative to"""
    hold(ask, [(a / 16, single(t), p, z) for a in range(1, 400, 3) for t in (0.5, 0.7, 0.75, 1.0, 1.3, 1.5, 3.0) for p in (32, 64, 100, 128, 394, 1000, 1024, 4097) for z in (0.0, 1e-30, -1e-30, 1e-18, -1e-18)])


def test_logits_at_edges(ask):
    rng = random.Random(3)
    cases = []
    for _ in range(4000):
        a, t, p = single(rng.choice([1, -1]) * 10.0 ** rng.uniform(-6, 6)), single(10.0 ** rng.uniform(-6, 6)), rng.choice([32, 64, 65536, rng.randint(32, 65536)])
        edge = a + rng.randint(-2816, 1280) * t / p
        cases += [(a, t, p, z) for z in near(single(edge), 2)]
    hold(ask, cases)

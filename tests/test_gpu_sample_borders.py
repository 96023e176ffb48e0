"""The choice of a word where its borders lie badly: at the edges of the bins that words are counted in, beyond what any word weighs, among millions of words that together weigh little beside one."""
import math

import pytest

torch = pytest.importorskip("torch")

import answering_reference as R  # noqa: E402
from paper_1807_05358_amd import operators as O  # noqa: E402
from test_gpu_sample import TYPES, check  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_min_p_that_no_word_reaches(t):
    """leaves the first word alone, of equal ones that of the lowest number: a few of them, hundreds, and more than are put in order"""
    z = torch.randn(8, 5003, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    z[0, 4:], z[0, :4] = -math.inf, torch.tensor([3.0, 5.0, 5.0, 1.0], device="cuda")
    z[1, 100:140] = 9.0
    z[2, ::10] = 9.0
    z[3, 7:] = 9.0
    z[4] = 0.0
    z[5, ::2], z[5, 1::2] = -0.0, 0.0
    z[6, 40:50] = math.inf
    z[7, 4000:4002] = 9.0
    z, u = z.to(TYPES[t]), torch.linspace(0.1, 0.99, 8, device="cuda")
    for min_p in (1.0 + 2.0 ** -23, 2.0, 1e30, torch.tensor([0.5, 1.0, 1.5, 7.0, 2.0, 1.0, 3.0, math.inf], device="cuda")):
        for parameters in (dict(), dict(top_p=0.9), dict(top_k=3), dict(top_k=4000, top_p=0.5), dict(temperature=0.2), dict(temperature=40.0, top_k=300)):
            words, logprob = check(z, u, min_p=min_p, **parameters)
            if not torch.is_tensor(min_p):
                assert int(words[0]) == 1 and float(logprob[0]) == 0.0
    z[3, 20] = math.nan
    z[4] = -math.inf
    words, logprob = check(z, u, min_p=2.0)
    assert words[3:5].tolist() == [-1, -1] and bool(torch.isnan(logprob[3:5]).all())


# temperature, largest logit and bins a unit, where the place of logit 0 is a rounding below a whole number: its bin ends at an edge that is 0, or a rounding below
EDGES = [(0.75, 0.5625, 2392), (0.75, 1.125, 1388), (0.75, 1.875, 776), (0.75, 2.625, 574), (0.75, 3.5625, 592), (0.75, 5.0625, 412), (0.75, 6.9375, 272), (1.5, 1.125, 2704), (1.5, 1.5, 2014), (1.5, 2.25, 1558),
         (1.5, 3.0, 1163), (1.5, 4.5, 773), (1.5, 6.0, 589), (3.0, 3.0, 2116), (3.0, 4.5, 1304), (3.0, 7.5, 1106)]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("each", [12, 300])
def test_logits_of_0_at_the_edge_of_a_bin(t, each):
    """words of logit 0, as many just above and as many just below decide, beside larger ones"""
    g = torch.Generator().manual_seed(each)
    cases = [(*e, part, what) for e in EDGES + [(0.5, 2.0, 333), (1.0, 3.0, 500)] for part in range(3) for what in ("u", "top_p")]
    step = 16 // torch.empty(0, dtype=TYPES[t]).element_size()                  # each thread of a row's block looks at so many words side by side
    z = torch.full((len(cases), 1024 * step), -math.inf, dtype=torch.float64)
    u, top_p = torch.full((len(cases),), 1 - 2.0 ** -24), torch.ones(len(cases))
    temperature = torch.tensor([c[0] for c in cases])
    for r, (T, top, per, part, what) in enumerate(cases):
        # the least of the threads' largest words, from which the bins' width is made
        apart = 704 / (per + 0.5) if per > 352 else (2816 / (per + 0.5) - 2) / 3
        z[r, ::step] = top - T * apart * torch.rand(1024, generator=g).double() / 2
        z[r, 0], z[r, step] = top, top - T * apart
        at = torch.randperm(1024, generator=g)[:3 * each] * step + 1
        beside = 1e-7 * (1 + torch.rand(each, generator=g).double())
        z[r, at[:each]], z[r, at[each:2 * each]], z[r, at[2 * each:]] = 0.0, -beside, beside
        z[r] = z[r].to(TYPES[t]).double()
        run = torch.exp((z[r] - top) / T).sort(descending=True)[0].cumsum(0)
        # in the middle of a word among those
        k = 1024 + part * each + each // 2
        (u if what == "u" else top_p)[r] = float((run[k] + run[k - 1]) / 2 / run[-1])
    check(z.to(TYPES[t]).cuda(), u.cuda(), temperature=temperature.cuda(), top_p=top_p.cuda())


def test_weights_that_are_1_in_64_bits():
    """at a high temperature words far below the largest weigh 1, too, and min_p of 1 or just below it leaves them: a few, and more than are put in order"""
    for V in (50, 1500, 9000):
        z = torch.randn(4, V, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")
        z[1] *= 1000
        z[2, ::3] = -math.inf
        u = torch.tensor([0.0, 0.3, 0.6, 0.97], device="cuda")
        for temperature in (1e20, 1e30, 3e38):
            for min_p in (1.0, 1 - 2.0 ** -24, 0.5):
                for parameters in (dict(), dict(top_k=40)):
                    check(z, u, temperature=temperature, min_p=min_p, **parameters)
                # half of equal words ends just where one of them does: both sums are to 2^-29 of themselves, so the border is to 2^-28, and the word behind it may be kept or not
                words, logprob = O.sample(z, u, temperature=temperature, min_p=min_p, top_p=0.5)
                for r, row in enumerate(z.cpu()):
                    may = [R.choose(row, float(u[r]), temperature, 0, 0.5 * (1 + side * 2.0 ** -28), min_p) for side in (-1, 0, 1)]
                    assert any(int(words[r]) == word and abs(float(logprob[r]) - log) <= 2.0 ** -24 * abs(log) + 1e-9 for word, log in may), (V, r, temperature, min_p, may, words[r], logprob[r])


@pytest.mark.parametrize("V", [1 << 14, 1 << 20, 1 << 24])
def test_many_words_that_weigh_little_each(V):
    """one word and V - 1 equal ones beside it, each of which may weigh less than 2^-38 of it and all of them 3e-5"""
    for t in (torch.float32, torch.bfloat16):
        z = torch.full((1, V), -math.log(V / 3e-5), device="cuda").to(t)
        at = V // 3
        z[0, at] = 0.0
        w = math.exp(float(z[0, 0]))
        total = 1 + (V - 1) * w
        for u in (0.5, 1 - 2.0 ** -15, 0.99999, 1 - 2.0 ** -18, 1 - 2.0 ** -24):
            u = float(torch.tensor(u, dtype=torch.float32))
            for top_p in (1.0, 0.99999):
                p = float(torch.tensor(top_p, dtype=torch.float32))
                n = V - 1 if top_p == 1.0 else math.ceil((p * total - 1) / w)       # of the equal words those that are kept
                left = 1 + n * w
                words, logprob = O.sample(z, torch.tensor([u], device="cuda"), top_p=top_p)
                k = math.floor((u * left - 1) / w)                                   # of them, those before the chosen one; below 0: the first word
                got = int(words[0])
                rank = -1 if got == at else got - (got > at)
                # sums to 2^-53 of themselves and of the largest word's weight a few times, and words rounded to 2^-79 of that, in words; and a word, of top_p and u each, where a border is next to one
                assert (rank == -1) == (k < 0) and abs(rank - max(k, -1)) <= 2 + (16 * 2.0 ** -53 + V * 2.0 ** -79) / w, (t, u, top_p, rank, k)
                want = math.log((1.0 if k < 0 else w) / left)
                assert abs(float(logprob[0]) - want) <= 2.0 ** -24 * abs(want) + 1e-9 + 2 * w


def test_sums_of_many_equal_words_beside_others():
    """a border of top_k, top_p or min_p among more equal words than are put in order, and words that weigh 2^-30 and less of the largest"""
    g = torch.Generator(device="cuda").manual_seed(4)
    z = torch.randn(4, 20011, generator=g, device="cuda")
    z[0, 1::4] = -19.0
    z[0, 0] = 9.0
    z[1, ::3] = -30.0
    z[1, 1::3] = -29.5
    z[1, 2::3] = -60.0
    z[1, 100] = 0.0
    z[2, ::2] = 1.0
    z[3, 5000:] = -3.0
    u = torch.tensor([1 - 2.0 ** -24, 1 - 2.0 ** -24, 0.7, 0.95], device="cuda")
    for parameters in (dict(), dict(top_k=9000), dict(top_k=15000, top_p=0.9), dict(min_p=1e-7), dict(top_p=0.99999994), dict(temperature=2.0), dict(temperature=0.7, top_p=0.99)):
        check(z, u, **parameters)

"""The choice of a word against its definition, row by row: whole numbers have to be equal."""
import math

import pytest

torch = pytest.importorskip("torch")

import answering_reference as R  # noqa: E402
from paper_1807_05358_amd import operators as O  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def check(z, u, **parameters):
    words, logprob = O.sample(z, u, **parameters)
    assert words.dtype == torch.int32 and logprob.dtype == torch.float32 and words.shape == u.shape == logprob.shape
    single = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    zc = z.cpu()
    for r in range(z.shape[0]):
        p = {n: (x[r].item() if torch.is_tensor(x) else x if n == "top_k" else single(x)) for n, x in parameters.items()}
        word, log = R.choose(zc[r], float(u[r]), **p)
        assert int(words[r]) == word, (r, p, float(u[r]), int(words[r]), word)
        # one rounding of a result in 64 bits, and the sums' steps of 2^-45 of the largest weight at least
        assert math.isnan(log) and math.isnan(float(logprob[r])) or abs(float(logprob[r]) - log) <= 2.0 ** -24 * abs(log) + 1e-9, (r, float(logprob[r]), log)
    return words, logprob


def rows(R_, V, t, spread=2.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (spread * torch.randn(R_, V, generator=g, device="cuda")).to(t), torch.rand(R_, generator=g, device="cuda")


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 1000, 1024, 1025, 4099, 20011])
def test_sizes_and_types(t, V):
    z, u = rows(6, V, TYPES[t], seed=V)
    check(z, u)
    check(z, u, temperature=0.6, top_k=5, top_p=0.8, min_p=0.02)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("parameters", [dict(temperature=0.0), dict(temperature=0.05), dict(temperature=5.0), dict(temperature=1e-3, top_k=40), dict(temperature=1e6), dict(top_k=1), dict(top_k=50), dict(top_k=3000), dict(top_k=10 ** 9), dict(top_k=-1),
                                        dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=0.1), dict(top_p=0.9), dict(top_p=0.9999), dict(top_p=1.0), dict(top_p=2.0), dict(min_p=0.1), dict(min_p=1.0), dict(min_p=7.0), dict(min_p=-1.0),
                                        dict(top_k=200, top_p=0.9), dict(top_k=200, min_p=0.01), dict(top_p=0.7, min_p=0.2), dict(top_p=0.99, min_p=1e-6), dict(top_k=30, top_p=0.95, min_p=0.05, temperature=1.3)])
def test_parameters(t, parameters):
    z, u = rows(12, 5003, TYPES[t], seed=len(str(parameters)))
    u[0], u[1], u[2] = 0.0, 1 - 2.0 ** -24, 0.5
    check(z, u, **parameters)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_ties(t):
    """equal logits are taken in the words' order, and any number of them may lie on a border"""
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randint(-2, 3, (10, 3001), generator=g, device="cuda").to(TYPES[t])
    z[0] = 1.0                                             # all alike
    z[1] = 0.0
    z[1, ::2] = -0.0
    z[2, 5:] = -math.inf
    u = torch.rand(10, generator=g, device="cuda")
    for parameters in (dict(), dict(top_k=700), dict(top_p=0.5), dict(top_k=1000, top_p=0.3), dict(min_p=0.5), dict(temperature=0.0), dict(top_p=0.25, min_p=0.9)):
        check(z, u, **parameters)
    check(z, torch.zeros_like(u), top_p=0.5)


def test_infinite_logits_and_rows_without_a_word():
    z, u = rows(9, 700, torch.float32)
    z[0, 100:] = -math.inf
    z[1] = -math.inf
    z[2, 3] = math.nan
    z[3, 50], z[3, 600] = math.inf, math.inf
    z[4, 699] = math.inf
    z[5] = -3e38
    z[6, 0] = 3e38
    z[7, :699] = -math.inf
    for parameters in (dict(), dict(temperature=0.0), dict(top_k=3, top_p=0.9), dict(min_p=0.1), dict(top_k=650)):
        words, logprob = check(z, u, **parameters)
        assert int(words[1]) == int(words[2]) == -1 and bool(torch.isnan(logprob[1:3]).all()) and int(words[4]) == 699 and int(words[7]) == 699


def test_random_numbers_outside_their_range():
    z, _ = rows(4, 300, torch.float32)
    u = torch.tensor([-1.0, -0.0, 1.0, 7.0], device="cuda")
    words, _ = O.sample(z, u, top_k=20)
    order = torch.sort(z, dim=1, descending=True, stable=True)[1]
    assert words.tolist() == [int(order[0, 0]), int(order[1, 0]), int(order[2, 19]), int(order[3, 19])]


def test_parameters_of_each_row():
    z, u = rows(8, 2000, torch.bfloat16)
    temperature = torch.tensor([1.0, 0.0, 0.5, -1.0, math.nan, math.inf, 2.0, 1e-30], device="cuda")
    top_k = torch.tensor([0, 5, 5, 5, 5, 5, 1, 100], device="cuda", dtype=torch.int32)
    top_p = torch.tensor([[0.9, 0], [0.9, 0], [0.5, 0], [1.0, 0], [1.0, 0], [1.0, 0], [0.3, 0], [1.0, 0]], device="cuda")[:, 0]      # strided
    words, logprob = check(z, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=0.01)
    assert words[3:6].tolist() == [-1, -1, -1]
    check(z, u, min_p=torch.linspace(0, 1, 8, device="cuda"), top_p=0.999)
    bad = torch.full((8,), math.nan, device="cuda")
    for p in (dict(top_p=bad), dict(min_p=bad)):
        assert O.sample(z, u, **p)[0].tolist() == [-1] * 8
    assert O.sample(z, bad)[0].tolist() == [-1] * 8


def test_strides_and_places():
    """rows inside wider ones, at any element's place; columns taken apart"""
    for t in TYPES.values():
        wide, u = rows(5, 3011, t, seed=3)
        for z in (wide[:, 1:3000], wide[:, 3:], wide[1:, :17], wide[:, ::3], wide.t()[:100].t(), wide[:1].expand(5, 3011)):
            check(z, u[:z.shape[0]], top_p=0.9)


def test_a_large_vocabulary():
    for t, V in ((torch.float32, 200003), (torch.bfloat16, 131072)):
        z, u = rows(3, V, t, seed=5)
        check(z, u)
        check(z, u, top_k=50, top_p=0.9)
        check(z, u, top_p=0.95)
        check(z, u, temperature=30.0, top_p=0.5, min_p=0.1)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_rows_that_are_read_again(t):
    """the largest logits far behind the first ones, and far above them; logits so far below the others that only a high temperature lets them count; a row whose first part is masked"""
    z, u = rows(6, 70000, TYPES[t], spread=1.0, seed=9)
    z[0, 60000:60050] += 60
    z[1, 69999] = 200.0
    z[2, 100:] -= 40
    z[3, ::3] -= 25
    z[4, :50000] = -math.inf
    z[5, 17:] = -math.inf
    for parameters in (dict(), dict(temperature=3.0, top_p=0.99), dict(temperature=9.0), dict(temperature=25.0, min_p=0.1), dict(temperature=0.1, top_k=60), dict(top_p=0.999, min_p=1e-7), dict(temperature=3.0, top_k=30000)):
        check(z, u, **parameters)


@pytest.mark.parametrize("t", ["f32", "f16"])
@pytest.mark.parametrize("spread", [0.003, 0.02, 0.1, 0.5])
def test_many_words_in_the_bins_that_decide(t, spread):
    """logits so near one another that dozens, hundreds or thousands of words have to be put in order"""
    z, u = rows(5, 9000, TYPES[t], spread=spread, seed=int(1000 * spread))
    for parameters in (dict(), dict(top_p=0.4), dict(top_k=4000, top_p=0.7), dict(min_p=0.99), dict(temperature=0.01, top_k=100)):
        check(z, u, **parameters)


def test_a_mask_that_leaves_a_few_words():
    z, u = rows(8, 50000, torch.bfloat16, seed=11)
    keep = torch.zeros(8, 50000, dtype=torch.bool, device="cuda")
    for r in range(8):
        keep[r, torch.randperm(50000, device="cuda")[:2 ** r]] = True
    z.masked_fill_(~keep, -math.inf)
    for parameters in (dict(), dict(temperature=4.0, top_p=0.5), dict(top_k=20), dict(temperature=0.0)):
        words, _ = check(z, u, **parameters)
        assert bool(keep.gather(1, words.long()[:, None]).all())


def test_shares_of_many_choices():
    """with every random number in turn, each word comes as often as its share says"""
    z = torch.randn(1, 40, device="cuda")
    n = 4000
    words, logprob = O.sample(z.expand(n, 40), (torch.arange(n, device="cuda") + 0.5) / n, temperature=0.8, top_p=0.9)
    share = torch.bincount(words.long(), minlength=40) / n
    want = torch.zeros(40, device="cuda")
    want[words.long()] = logprob.exp()
    assert float((share - want).abs().max()) <= 1.01 / n and abs(float(want.sum()) - 1) < 1e-5


def test_captured_and_replayed():
    z, u = rows(4, 3000, torch.float32)
    out = O.sample(z, u, top_p=0.9)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = O.sample(z, u, top_p=0.9)
    for seed in range(4):
        a, b = rows(4, 3000, torch.float32, seed=seed)
        z.copy_(a), u.copy_(b)
        g.replay()
        got = [x.clone() for x in out]
        want = O.sample(z, u, top_p=0.9)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_requires_grad_is_refused():
    z, u = rows(2, 30, torch.float32)
    z.requires_grad_()
    with pytest.raises(ValueError):
        O.sample(z, u)
    with torch.no_grad():
        O.sample(z, u)


def test_as_many_rows_and_words_as_there_may_be():
    torch.manual_seed(11)
    # every row of two words: the larger one weighs 1 of 1 + e^-d
    R_, u = (1 << 22) - 1, torch.rand((1 << 22) - 1, device="cuda")
    z = torch.randn(R_, 2, device="cuda").half()
    words, logprob = O.sample(z, u)
    first = (z[:, 1] > z[:, 0]).int()
    share = 1 / (1 + torch.exp(-(z[:, 0].double() - z[:, 1].double()).abs()))
    near = (u.double() - share).abs() < 1e-8
    want = torch.where(u.double() < share, first, 1 - first)
    assert bool(((words == want) | near).all())
    p = torch.where(words == first, share, 1 - share)
    assert float((logprob.double() - p.log()).abs().max()) < 1e-6
    # 2^24 words, with and without many equal ones
    for t in (torch.float32, torch.float16):
        z, u = torch.randn(2, 1 << 24, device="cuda").to(t), torch.tensor([0.3, 0.999], device="cuda")
        words, logprob = O.sample(z, u, temperature=0.5, top_p=0.7)
        for row in range(2):
            w = torch.exp((z[row].double() - z[row].double().max()) / 0.5)
            order = torch.sort(z[row], descending=True, stable=True)[1]
            run = torch.cumsum(w[order], 0)
            n = int(torch.searchsorted(run, 0.7 * run[-1])) + 1
            at = int((order == words[row]).nonzero()[0])
            target = float(u[row]) * float(run[n - 1])
            # the sums: to 2^-29 of themselves, and where top_p cuts by a word, 2e-6 of all, more or less
            slack = 1e-8 * target + float(w[order[n - 1]])
            assert float(run[at] - w[words[row]]) - slack <= target <= float(run[at]) + slack
            assert abs(float(logprob[row]) - math.log(float(w[words[row]] / run[n - 1]))) < 1e-5


def test_on_two_streams_at_once():
    z, u = rows(64, 30000, torch.bfloat16)
    want = [O.sample(z, u, top_p=p) for p in (0.5, 0.95)]
    streams = [torch.cuda.Stream() for _ in want]
    got = []
    for s, p in zip(streams, (0.5, 0.95)):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([O.sample(z, u, top_p=p) for _ in range(5)])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, several in zip(want, got) for g in several for x, y in zip(g, w))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("top_k", [1, 2, 63, 64, 65, 128, 129, 255, 256, 257])
def test_the_first_words(t, top_k):
    """rows in whose order the words of top_k lie badly: in turn, all in one thread's share, more alike than are put in order, fewer than top_k, an infinite one"""
    V = 70001
    z, u = rows(10, V, TYPES[t], seed=top_k)
    z[1], z[2] = z[1].sort()[0], z[2].sort(descending=True)[0]
    for base in range(40, V - 8, 8192):                     # of one thread, whatever it takes at once
        z[3, base:base + 8] = 20 + torch.randn(8, device="cuda").to(z.dtype)
    z[4, 100:5000] = 15.0
    z[5], z[6] = 0.25, -math.inf
    z[6, ::600] = torch.randn(len(z[6, ::600]), device="cuda").to(z.dtype)
    z[7, 69000] = math.inf
    z[8, 69999] = math.nan
    z[9, :] = -3e38
    z[9, 5:70] = 3e38
    for parameters in (dict(), dict(top_p=0.8), dict(min_p=0.3), dict(temperature=40.0, top_p=0.5, min_p=0.01), dict(temperature=0.01)):
        check(z, u, top_k=top_k, **parameters)


@pytest.mark.parametrize("spread", [0.1, 1.0, 6.0])
def test_the_words_of_min_p(spread):
    """few and many of them, those next to the border among them"""
    z, u = rows(6, 30000, torch.float32, spread=spread, seed=5)
    z[1, 7] = z[1].max() + 3
    z[2, :3000] = z[2].max()
    top = z[3].max()
    for i, f in enumerate((0.05, 0.0499, 0.0501, 0.02)):
        z[3, 100 * i] = top + math.log(f)
    for min_p in (0.0157, 0.02, 0.05, 0.3, 1.0):
        check(z, u, min_p=min_p)
        check(z, u, min_p=min_p, top_k=100, temperature=2.0)


def test_flat_rows():
    """logits a thousandth apart, and rows of two parts far from one another"""
    for V, spread in ((40000, 1e-3), (150000, 0.05)):
        z, u = rows(3, V, torch.float32, spread=spread, seed=7)
        z[1, V // 2:] -= 30
        z[2, 17:] -= 5
        for parameters in (dict(), dict(top_p=0.9), dict(top_k=5000, top_p=0.9), dict(temperature=3.0, min_p=0.9)):
            check(z, u, **parameters)

"""The operators that a decoder answers with, together: prompts of different lengths, single tokens and several at once from one cache, against the same model in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import language_model as L, operators as O  # noqa: E402

pytestmark = pytest.mark.gpu
VOCAB, HIDDEN, HEADS, LAYERS = 301, 128, 2, 2


def plain_logits(model, tokens):
    """behind the last of one sequence's tokens, in 64 bits"""
    p = {k: v.double() for k, v in model.params.items()}
    h = p["embedding"][tokens.long()]
    S, D = h.shape

    def norm(x, name):
        m = x.mean(1, keepdim=True)
        v = ((x - m) ** 2).mean(1, keepdim=True)
        return (x - m) / torch.sqrt(v + 1e-5) * p[name + ".w"] + p[name + ".b"]

    for n in range(model.layers):
        q, k, v = (norm(h, f"{n}.a") @ p[f"{n}.qkv"].t()).view(S, 3, HEADS, D // HEADS).permute(1, 2, 0, 3).unbind()
        z = (q @ k.transpose(1, 2)) * (D // HEADS) ** -0.5
        z = z.masked_fill(torch.ones(S, S, device=z.device, dtype=torch.bool).triu(1), -math.inf)
        h = h + (torch.softmax(z, 2) @ v).transpose(0, 1).reshape(S, D) @ p[f"{n}.out"].t()
        h = h + torch.relu(norm(h, f"{n}.b") @ p[f"{n}.up"].t()) @ p[f"{n}.down"].t()
    return (norm(h, "last") @ p["words"].t())[-1]


def prompts(batch, length, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, VOCAB, (batch, length), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("few", [L.Cache.FEW, 8])
@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
def test_extend_in_any_pieces(t, few):
    """a prompt, then a piece, from the pages or read back, then few tokens, then single ones: behind each, the logits of all that came before"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=t, seed=1)
    tokens = prompts(3, 80)
    cache = L.Cache(model, 3, 80, page=16)
    cache.FEW = few
    had = [[], [], []]
    # rounding of about 15 tensors in each layer and 10 outside, each at most half a step of its size
    most = (15 * LAYERS + 10) * torch.finfo(t).eps / 2
    at = 0
    for piece, lengths in ((40, [40, 13, 1]), (20, [20, 20, 7]), (5, [5, 2, 5]), (1, [1, 1, 1]), (8, [3, 8, 1]), (1, [1, 1, 1])):
        new = tokens[:, at:at + piece]
        at += piece
        logits = model.extend(cache, new, torch.tensor(lengths, dtype=torch.int32, device="cuda"))
        for b in range(3):
            had[b] += new[b, :lengths[b]].tolist()
            want = plain_logits(model, torch.tensor(had[b], device="cuda"))
            assert (logits[b].double() - want).norm() <= most * want.norm(), (b, piece)
    assert cache.lengths.tolist() == [len(x) for x in had] and cache.filled == 75
    with pytest.raises(ValueError):
        model.extend(cache, tokens[:, :6])


@pytest.mark.parametrize("held,steps", [("e4m3", 2.0 ** -4), ("e2m1", 2.0 ** -2)])
def test_a_cache_in_fewer_bits(held, steps):
    """the logits move by no more than the keys' and values' own roundings let them, and choose as the model with those keys and values would"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, seed=2)
    tokens = prompts(2, 50, seed=3)
    whole, less = L.Cache(model, 2, 64), L.Cache(model, 2, 64, held=held)
    a, b = model.extend(whole, tokens), model.extend(less, tokens)
    # half a step relative to each value, a layer's softmax and sums once each
    assert (a - b).norm() <= LAYERS * 2 * steps * a.norm()
    # from pages and read back alike: the contiguous kernel rounds its probabilities, half a step
    for n in range(LAYERS):
        pages, scales = less.layer(n)
        q = torch.randn(2, HEADS, 4, HIDDEN // HEADS, device="cuda").bfloat16()
        o, _ = O.attention_paged_fwd(q, *pages, less.table, less.lengths, causal=True, **scales)
        k, v = O.cache_read(*pages, less.table, less.lengths, kv_len=50, dtype=torch.bfloat16, **scales)
        r, _ = O.attention_fwd(q, k, v, causal=True)
        assert float((o.double() - r.double()).abs().max()) <= 3 * 2.0 ** -8 * float(v.double().abs().max())


def test_generate():
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.float16, seed=4)
    tokens = prompts(4, 30, seed=5)
    lengths = torch.tensor([30, 1, 17, 30], dtype=torch.int32, device="cuda")
    u = torch.rand(4, 12, device="cuda")
    words, logprob = model.generate(L.Cache(model, 4, 48), tokens, u, lengths, temperature=0.8, top_k=40, top_p=0.9)
    assert words.shape == logprob.shape == (4, 12) and bool(((words >= 0) & (words < VOCAB)).all()) and bool((logprob <= 0).all())
    again = model.generate(L.Cache(model, 4, 48, page=16), tokens, u, lengths, temperature=0.8, top_k=40, top_p=0.9)
    assert torch.equal(again[0], words)
    # the most likely words, without random numbers: as the whole sequence in 64 bits has them, unless two logits are nearer than roundings
    greedy, _ = model.generate(L.Cache(model, 4, 48), tokens, u, lengths, temperature=0.0)
    most = (15 * LAYERS + 10) * 2.0 ** -11
    for b in range(4):
        for i in (0, 5, 11):
            z = plain_logits(model, torch.cat([tokens[b, :lengths[b]], greedy[b, :i]]))
            assert float(z.max() - z[greedy[b, i].long()]) <= 2 * most * float(z.norm())


def test_a_step_in_a_graph():
    """one token of each sequence, captured: the graph moves the lengths itself"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, seed=6)
    tokens = prompts(2, 20, seed=7)
    u = torch.rand(2, 10, device="cuda")
    want, _ = model.generate(L.Cache(model, 2, 64), tokens, u, top_p=0.9)
    cache = L.Cache(model, 2, 64)
    word = O.sample(model.extend(cache, tokens), u[:, 0].contiguous(), top_p=0.9)[0]
    got = [word.clone()]
    now, length, number = word.clone(), cache.lengths.clone(), u[:, 1].clone()

    def step():
        cache.lengths = length
        out = O.sample(model.extend(cache, now[:, None]), number, top_p=0.9)[0]
        length.copy_(cache.lengths)
        now.copy_(out)

    saved = [x.clone() for x in (now, length)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    now.copy_(saved[0]), length.copy_(saved[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(1, 10):
        number.copy_(u[:, i])
        g.replay()
        got.append(now.clone())
    assert torch.equal(torch.stack(got, 1), want)


def test_a_call_that_fails_leaves_the_cache_as_it_was():
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, seed=8)
    tokens = prompts(2, 20, seed=9)
    cache = L.Cache(model, 2, 64)
    model.extend(cache, tokens)
    for bad in (lambda: model.extend(cache, prompts(3, 4)), lambda: model.extend(cache, tokens, torch.ones(2, dtype=torch.int64, device="cuda")), lambda: model.extend(cache, tokens[:, :0]),
                lambda: model.generate(cache, tokens, torch.rand(2, 26, device="cuda")), lambda: model.generate(cache, tokens, torch.rand(2, 0, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    assert cache.filled == 20 and cache.lengths.tolist() == [20, 20]


def test_lengths_beyond_the_new_tokens():
    """are those of all of them: nothing behind them is looked at"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, seed=8)
    tokens = prompts(2, 20, seed=9)
    a, b = L.Cache(model, 2, 64), L.Cache(model, 2, 64)
    for new in (tokens, tokens[:, :3]):
        x, y = model.extend(a, new), model.extend(b, new, torch.tensor([10 ** 6, new.shape[1]], dtype=torch.int32, device="cuda"))
        assert torch.equal(x, y) and a.lengths.tolist() == b.lengths.tolist()


@pytest.mark.parametrize("piece", [1, 4, 9])
def test_a_captured_piece_moves_the_lengths(piece):
    """replayed as it stands, pieces of a sequence one behind the other: few tokens from the pages, more by way of reading back"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.float16, seed=10)
    tokens = prompts(2, 11 + 4 * piece, seed=11)
    eager, cache = L.Cache(model, 2, 64, page=16), L.Cache(model, 2, 64, page=16)
    eager.FEW = cache.FEW = 8
    model.extend(eager, tokens[:, :11]), model.extend(cache, tokens[:, :11])
    new = tokens[:, 11:11 + piece].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        model.extend(L.Cache(model, 2, 64, page=16), new)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = model.extend(cache, new)
    assert cache.filled == 11
    for at in range(11, 11 + 4 * piece, piece):
        new.copy_(tokens[:, at:at + piece])
        g.replay()
        want = model.extend(eager, new)
        assert cache.lengths.tolist() == eager.lengths.tolist() == [at + piece] * 2
        # kernels of another number of keys may add in another order: a rounding of each of the layers' outputs
        assert (got - want).norm() <= (15 * LAYERS + 10) * 2.0 ** -11 * want.norm()

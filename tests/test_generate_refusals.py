"""Decoder.generate refuses random numbers and a choice that it cannot take before the cache holds any of the tokens."""
import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import language_model as L  # noqa: E402

VOCAB, HIDDEN, HEADS, LAYERS = 61, 64, 1, 1


def calls(device):
    """(error, its words, u, choice) that no call of two sequences takes"""
    u = torch.rand(2, 3, device=device)
    return [(ValueError, "u has shape", u[:1], {}), (ValueError, "u has shape", torch.rand(3, 3, device=device), {}), (ValueError, "u is", u.double(), {}), (ValueError, "matrices", u[0], {}),
            (ValueError, "temperature is", u, dict(temperature=-1.0)), (ValueError, "temperature is", u, dict(temperature=float("nan"))), (ValueError, "top_p is", u, dict(top_p=float("inf"))),
            (ValueError, "min_p is", u, dict(min_p=float("nan"))), (ValueError, "32 bits", u, dict(top_k=1 << 31)), (ValueError, "top_k is torch.int64", u, dict(top_k=torch.ones(2, dtype=torch.int64, device=device))),
            (ValueError, "min_p has shape", u, dict(min_p=torch.ones(3, device=device))), (ValueError, "temperature is torch.float16", u, dict(temperature=torch.ones(2, dtype=torch.float16, device=device))),
            (ValueError, "gradients", u, dict(top_p=torch.ones(2, device=device, requires_grad=True))), (TypeError, "top", u, dict(top=3))]


def test_refusals_come_before_the_work():
    """on the CPU, where extend could not even begin"""
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, device="cpu")
    tokens = torch.zeros(2, 5, dtype=torch.int32)
    for error, words, u, choice in calls("cpu"):
        with pytest.raises(error, match=words):
            model.generate(L.Cache(model, 2, 32, device="cpu"), tokens, u, **choice)
    with pytest.raises(ValueError, match="matrices"):
        model.generate(L.Cache(model, 2, 32, device="cpu"), tokens[0], torch.rand(2, 3))


@pytest.mark.gpu
def test_a_refused_call_leaves_the_cache_as_it_was():
    model = L.Decoder(VOCAB, HIDDEN, HEADS, LAYERS, dtype=torch.bfloat16, seed=3)
    tokens = torch.randint(0, VOCAB, (2, 5), device="cuda", dtype=torch.int32)
    cache, other = L.Cache(model, 2, 32), L.Cache(model, 2, 32)
    for c in (cache, other):
        model.extend(c, tokens)
    for error, words, u, choice in calls("cuda") + [(ValueError, "u is on", torch.rand(2, 3), {}), (ValueError, "min_p is on", torch.rand(2, 3, device="cuda"), dict(min_p=torch.ones(2)))]:
        with pytest.raises(error, match=words):
            model.generate(cache, tokens, u, **choice)
        assert cache.filled == 5 and cache.lengths.tolist() == [5, 5]
    u = torch.rand(2, 4, device="cuda")
    assert all(torch.equal(x, y) for x, y in zip(model.generate(cache, tokens, u, top_p=0.9), model.generate(other, tokens, u, top_p=0.9)))

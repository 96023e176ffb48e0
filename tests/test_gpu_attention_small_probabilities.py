"""Attention where thousands of probabilities far below the row's largest make up the output."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_1807_05358_amd import operators
    return operators


def normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * scale


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("gap", [10.0, 14.0, 16.0, 17.0, 17.5, 19.0])
@pytest.mark.parametrize("B,H,K,Sq,n,D", [(1, 2, 1, 40, 4096, 64), (2, 4, 1, 1, 16000, 128), (1, 1, 1, 300, 1000, 80)])
def test_probabilities_far_below_the_largest(ops, B, H, K, Sq, n, D, gap, dtype):
    """a first key that takes nearly all of the probability and has no value: what is left is the sum of thousands of small ones"""
    g = gen(int(gap * 10) + n)
    q, k, v = normal(g, B, H, Sq, D, scale=0.3), normal(g, B, K, n, D, scale=0.3), 1 + normal(g, B, K, n, D, scale=0.3)
    q[..., 0], k[..., 0], v[:, :, 0] = 8.0, 0.0, 0.0
    k[:, :, 0, 0] = gap * math.sqrt(D) / 8
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    o, lse = ops.attention_fwd(q, k, v)
    want = R.attention_fwd(q, k, v)
    R.close(lse, *want["lse"], "lse")
    # the reference's bound without its term for what leaves the type's exponents; that is, in float16, half a step of 2^-32 of the row's largest probability (2^8 times the
    # probabilities are rounded) for every key
    value, bound = want["o"]
    bound = bound - R.tiny(dtype) * (n / 256)
    p = R._attention(q, k, v, False, None, None, D ** -0.5)[5]
    if dtype == F16:
        bound = bound + 1.01 * 2.0 ** -33 * p.amax(3, keepdim=True) * v.double().abs().sum(2, keepdim=True).repeat_interleave(H // K, 1)
    R.close(o, value, bound, "o")

"""Tensors whose elements lie more than 2^32 bytes from their start."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_1807_05358_amd import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=BF16)


def test_attention_over_a_long_cache(ops):
    """2.4 million positions of 8 heads: 4.9 GB of keys, the last heads and positions beyond 2^32 bytes"""
    g = gen(1)
    S, H, D = 2_400_003, 8, 128
    k, v = normal(g, 1, S, H, D).transpose(1, 2), normal(g, 1, S, H, D).transpose(1, 2)
    q, dout = normal(g, 1, H, 3, D), normal(g, 1, H, 3, D)
    o, lse = ops.attention_fwd(q, k, v, causal=True)
    dq, dk, dv = ops.attention_bwd(dout, q, k, v, o, lse, causal=True)
    for h in (0, 7):
        one = slice(h, h + 1)
        want = R.attention_fwd(q[:, one], k[:, one], v[:, one], causal=True)
        R.close(o[:, one], *want["o"], "o")
        R.close(lse[:, one], *want["lse"], "lse")
        want, _, _ = R.attention_bwd(dout[:, one], q[:, one], k[:, one], v[:, one], causal=True)
        # o, as the forward pass made it, is off by the rounding of the probabilities, too, which is not in the reference's delta
        p = torch.softmax(D ** -0.5 * q[:, one].double() @ k[:, one].double().transpose(2, 3), 3)
        off = R.half(BF16) * p * (p * (dout[:, one].double() @ v[:, one].double().transpose(2, 3)).abs()).sum(3, keepdim=True)
        R.close(dq[:, one], want["dq"][0], want["dq"][1] + 1.01 * D ** -0.5 * off @ k[:, one].double().abs(), "dq")
        R.close(dk[:, one], want["dk"][0], want["dk"][1] + 1.01 * D ** -0.5 * off.transpose(2, 3) @ q[:, one].double().abs(), "dk")
        R.close(dv[:, one], *want["dv"], "dv")


def test_layernorm_and_vocab_loss_of_many_elements(ops):
    """300007 rows of 8192 elements, 4.9 GB"""
    g = gen(2)
    N, D, V = 300_007, 8192, 70
    x, w, b = normal(g, N, D), normal(g, D), normal(g, D)
    last = slice(N - 300, N)
    y, h, mean, rstd = ops.layernorm_fwd(x, w, b)
    for (name, (value, bound)), z in zip(R.layernorm_fwd(x[last], w, b, None, 1e-5).items(), (y, h, mean, rstd)):
        R.close(z[last], value, bound, name)
    dx = ops.layernorm_bwd(y, h, w, mean, rstd, dh=x)[0]
    R.close(dx[last], *R.layernorm_bwd(y[last], h[last], w, mean[last], rstd[last], x[last])["dx"], "dx")
    del y, dx
    words = normal(g, V, D) * (1.5 / math.sqrt(D))
    t = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    t[::3] = -100
    got = ops.vocab_loss_fwd(x, words, t)
    for (name, (value, bound)), z in zip(R.vocab_loss_fwd(x[last], words, t[last]).items(), got):
        R.close(z[last], value, bound, name)
    dloss = torch.ones(N, device="cuda")
    dx = ops.vocab_loss_bwd(dloss, x, words, t, got[1])[0]
    R.close(dx[last], *R.vocab_loss_bwd(dloss[last], x[last], words, t[last], got[1][last])["dx"], "dx")


def test_rows_far_apart(ops):
    """strides of 2^24 elements and more: 64 rows of a tile are 2 GB apart, which the loads of whole tiles do not reach"""
    g = gen(3)
    S, D, wide = 150, 64, (1 << 24) + 8
    big = torch.zeros(S, wide, device="cuda", dtype=BF16)           # 5 GB
    k, v, q, dout = (big[:, at:at + D] for at in (0, D, 2 * D, wide - D))
    for m in (k, v, q, dout):
        m.copy_(normal(g, S, D))
    k, v, q, dout = (m[None, None] for m in (k, v, q, dout))
    for causal in (False, True):
        want, o, lse = R.attention_bwd(dout, q, k, v, causal=causal)
        for (name, (value, bound)), got in zip(R.attention_fwd(q, k, v, causal=causal).items(), ops.attention_fwd(q, k, v, causal=causal)):
            R.close(got, value, bound, name)
        for (name, (value, bound)), got in zip(want.items(), ops.attention_bwd(dout, q, k, v, o.to(BF16), lse.float(), causal=causal)):
            R.close(got, value, bound, name)
    x, w = q[0, 0], k[0, 0]
    t = torch.randint(0, S, (S,), generator=g, device="cuda", dtype=torch.int32)
    got = ops.vocab_loss_fwd(x, w, t)
    for (name, (value, bound)), z in zip(R.vocab_loss_fwd(x, w, t).items(), got):
        R.close(z, value, bound, name)
    dloss = torch.ones(S, device="cuda")
    for (name, (value, bound)), z in zip(R.vocab_loss_bwd(dloss, x, w, t, got[1]).items(), ops.vocab_loss_bwd(dloss, x, w, t, got[1])):
        R.close(z, value, bound, name)
    weight = normal(g, D)
    for (name, (value, bound)), z in zip(R.layernorm_fwd(x, weight, None, w, 1e-5).items(), ops.layernorm_fwd(x, weight, residual=w)):
        R.close(z, value, bound, name)

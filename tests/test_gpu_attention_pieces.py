"""Attention's backward pass where the call's keys hold nearly all of a row's probability, and the rest of it, with much larger values, is another call's."""
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


def case(dtype, m, size, first, rest, Sq=40, D=64):
    """keys 0 .. first-1: one that all rows look at and others that none does; then `rest` keys of 2^-m of a row's probability in all, with values `size` times as large"""
    g = torch.Generator(device="cuda")
    g.manual_seed(m * 100 + first)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    q, k, v, dout = normal(1, 4, Sq, D, scale=0.1), normal(1, 2, first + rest, D, scale=0.1), normal(1, 2, first + rest, D), normal(1, 4, Sq, D)
    q[..., 0] = 8.0                     # times 1 / sqrt(D): scores are the keys' first element
    k[:, :, :first, 0] = -30.0
    k[:, :, first - 1, 0] = math.log(rest * 2.0 ** m)
    k[:, :, first:, 0] = 0.0
    v[:, :, first:] *= size
    return [x.to(dtype) for x in (dout, q, k, v)]


@pytest.mark.parametrize("dtype,m,size", [(BF16, 11, 250), (BF16, 12, 500), (BF16, 13, 1000), (BF16, 16, 8000), (BF16, 18, 30000),
                                          (F16, 11, 40), (F16, 12, 80), (F16, 13, 160), (F16, 16, 1300), (F16, 18, 5000)])
@pytest.mark.parametrize("first", [1, 3, 64, 100])
def test_piece_with_nearly_all_of_the_probability(ops, dtype, m, size, first):
    rest = 8
    dout, q, k, v = case(dtype, m, size, first, rest)
    want, o, lse = R.attention_bwd(dout, q, k, v)
    n = first + rest
    parts = [ops.attention_bwd(dout, q, k[:, :, a:b], v[:, :, a:b], o.to(dtype), lse.float()) for a, b in ((0, first), (first, n))]
    # the reference's bounds have one rounding of o in delta.  Where the piece's own sum of p dp stands for <do, o>, it is as far from it as that rounding and one
    # of the probabilities can be at most, so delta is off by another rounding of o and one of p.
    scale = q.shape[3] ** -0.5
    kd, vd = (x.double().repeat_interleave(2, 1) for x in (k, v))
    p = torch.softmax(scale * q.double() @ kd.transpose(2, 3), 3)
    do = dout.double()
    off = R.half(dtype) * ((do * (p @ vd)).abs().sum(3, keepdim=True) + (p * (do @ vd.transpose(2, 3))).abs().sum(3, keepdim=True))
    more_q = 1.01 * scale * (p * off) @ kd.abs()
    more_k = 1.01 * (scale * (p * off).transpose(2, 3) @ q.double().abs()).reshape(1, 2, 2, n, -1).sum(2)
    dq = parts[0][0].double() + parts[1][0].double()
    R.close(dq, want["dq"][0], want["dq"][1] + more_q + R.half(dtype) * sum(x[0].double().abs() for x in parts) + R.tiny(dtype), "dq")
    R.close(torch.cat([x[1] for x in parts], 2), want["dk"][0], want["dk"][1] + more_k, "dk")
    R.close(torch.cat([x[2] for x in parts], 2), *want["dv"], "dv")

"""Attention in float16 where its exponents end: values that take dp out of them."""
import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

F16 = torch.float16


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


#       B  H  K  Sq  Sk    D    causal
LARGE = [(1, 2, 1, 40, 3, 128, False), (2, 4, 2, 33, 8, 128, True), (1, 2, 2, 70, 300, 128, False), (1, 4, 1, 130, 200, 64, True), (1, 1, 1, 20, 4096, 128, False),
         (1, 8, 1, 1, 70, 80, False), (3, 2, 2, 65, 65, 32, True)]


@pytest.mark.parametrize("size", [30, 500, 4000, 20000])
@pytest.mark.parametrize("case", LARGE, ids=lambda c: "-".join(str(x) for x in c))
def test_gradients_with_large_values(ops, case, size):
    """values whose products with the gradient are up to dim times as large as it: dp of some keys is 2^7 times 20000 |do|, and the gradients are finite"""
    B, H, K, Sq, Sk, D, causal = case
    g = gen(Sq * 1000 + Sk + size)
    q, k = normal(g, B, H, Sq, D).to(F16), normal(g, B, K, Sk, D).to(F16)
    along = torch.sign(normal(g, 1, 1, 1, D))
    v = (size * along * torch.sign(normal(g, B, K, Sk, 1)) * (1 + normal(g, B, K, Sk, D, scale=0.1)).clamp(0.5, 1.5)).to(F16)
    dout = (along * normal(g, B, H, Sq, 1) * (1 + normal(g, B, H, Sq, D, scale=0.1)) / size).to(F16)
    want, o, lse = R.attention_bwd(dout, q, k, v, causal=causal)
    assert all(torch.isfinite(x.to(F16)).all() for x, _ in want.values())
    got = ops.attention_bwd(dout, q, k, v, o.to(F16), lse.float(), causal=causal)
    # ds is rounded relative to its size but for what is below the type's exponents: half a step of 2^-24 times the unit that it is kept relative to.  The reference has the
    # largest |do| for that; with these values it is up to 2^10 times that of the row for dq, and for dk 2^-14 of the largest that ds can be.
    G, scale = H // K, D ** -0.5
    p = (R._attention(q, k, v, causal, None, None, scale)[5] > 0).double()
    do, vd = dout.double(), v.double().repeat_interleave(G, 1)
    unit_q = 1024 * do.abs().amax(3, keepdim=True)
    most = do.norm(dim=3).amax(2, keepdim=True)[..., None] * vd.norm(dim=3).amax(2, keepdim=True)[..., None] * 2
    unit_k = (most * 2.0 ** -14).view(B, K, G, 1, 1).amax(2).repeat_interleave(G, 1)
    b_q = 1.01 * scale * (p * R.tiny(F16) * unit_q) @ k.double().abs().repeat_interleave(G, 1)
    b_k = 1.01 * scale * ((p * R.tiny(F16) * unit_k).transpose(2, 3) @ q.double().abs()).reshape(B, K, G, Sk, D).sum(2)
    R.close(got[0], want["dq"][0], want["dq"][1] + b_q, "dq")
    R.close(got[1], want["dk"][0], want["dk"][1] + b_k, "dk")
    R.close(got[2], *want["dv"], "dv")
    for a, b in zip(got, ops.attention_bwd(dout, q, k, v, o.to(F16), lse.float(), causal=causal)):
        assert torch.equal(a, b)


def test_large_values_of_one_key_leave_the_other_keys_their_precision(ops):
    """dk of a key with small values is as precise as without the large ones of a key that no query looks at"""
    g = gen(77)
    q, k, v, dout = (normal(g, 1, 2, 90, 64).to(F16) for _ in range(4))
    q[..., 0] = 8.0
    k[:, :, 40, 0] = -60.0              # exp(-60): nothing of it is left
    plain = R.attention_bwd(dout, q, k, v)
    v[:, :, 40] = 30000.0
    want, o, lse = R.attention_bwd(dout, q, k, v)
    got = ops.attention_bwd(dout, q, k, v, o.to(F16), lse.float())
    R.close(got[0], *want["dq"], "dq")
    for n, name in ((1, "dk"), (2, "dv")):
        others = torch.arange(90, device="cuda") != 40
        R.close(got[n][:, :, others], plain[0][name][0][:, :, others], plain[0][name][1][:, :, others], name)

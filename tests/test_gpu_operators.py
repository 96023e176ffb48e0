"""The training operators against their definitions in 64 bits, at the sizes, strides and masks where they can go wrong.
Bounds are those of operators_reference.py: half a step of the type for every rounding that include/ff_ops.h names, and the
additions of the sums."""
import math

import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_1807_05358_amd import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, to=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(to)


def compare(got, want):
    for (name, (value, bound)), x in zip(want.items(), got):
        R.close(x, value, bound, name)


# ---- layer norm ------------------------------------------------------------------------

LN = [(1, 1), (1, 8), (3, 7), (5, 64), (64, 1024), (7, 513), (130, 520), (33, 1001), (9, 2048), (6, 2049), (4, 4096), (5, 8192), (3, 8200), (2, 16384), (3, 20001), (2, 32768), (1, 65536), (1, 65535)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols", LN)
def test_layernorm(ops, dtype, rows, cols):
    g = gen(rows * 70000 + cols)
    x = normal(g, rows, cols, to=dtype) + normal(g, rows, 1, to=dtype)
    w, b = normal(g, cols, to=dtype), normal(g, cols, to=dtype)
    for res, bias in ((None, b), (normal(g, rows, cols, to=dtype), None)):
        got = ops.layernorm_fwd(x, w, bias, residual=res, eps=1e-5)
        compare(got, R.layernorm_fwd(x, w, bias, res, 1e-5))
        _, h, mean, rstd = got
        dy, dh = normal(g, rows, cols, to=dtype), None if res is None else normal(g, rows, cols, to=dtype)
        compare(ops.layernorm_bwd(dy, h, w, mean, rstd, dh=dh), R.layernorm_bwd(dy, h, w, mean, rstd, dh))


@pytest.mark.parametrize("rows,cols", [(3000, 96), (2100, 2500), (40001, 16), (5000, 1024)])
def test_layernorm_weight_gradients_of_many_rows(ops, rows, cols):
    g = gen(rows)
    for dtype in (F32, BF16):
        h, dy, w = normal(g, rows, cols, to=dtype), normal(g, rows, cols, to=dtype), normal(g, cols, to=dtype)
        _, _, mean, rstd = ops.layernorm_fwd(h, w)
        first = ops.layernorm_bwd(dy, h, w, mean, rstd)
        compare(first, R.layernorm_bwd(dy, h, w, mean, rstd, None))
        for a, b in zip(first, ops.layernorm_bwd(dy, h, w, mean, rstd)):
            assert torch.equal(a, b)


def test_layernorm_strides(ops):
    """rows that are slices, repeated rows, elements that do not lie side by side"""
    g = gen(5)
    for wide, cols, at in ((200, 64, 3), (200, 64, 8), (333, 100, 1)):
        big = normal(g, 17, wide, to=BF16)
        x, res = big[:, at:at + cols], normal(g, 1, cols, to=BF16).expand(17, cols)
        w, b = normal(g, cols + 1, to=BF16)[1:], normal(g, cols, to=BF16)
        compare(ops.layernorm_fwd(x, w, b, residual=res), R.layernorm_fwd(x, w, b, res, 1e-5))
        y, h, mean, rstd = ops.layernorm_fwd(x, w, b)
        dy = normal(g, cols, 17, to=BF16).t()
        compare(ops.layernorm_bwd(dy, h, w, mean, rstd, dh=res), R.layernorm_bwd(dy, h, w, mean, rstd, res))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cols", [2, 3, 5, 9, 12, 15, 77, 127, 128, 129, 255, 645, 1025, 2433, 4097, 5811, 14233])
def test_layernorm_rows_of_any_length_and_place(ops, cols, dtype):
    """rows that start at any element: the last lanes' accesses overlap those before, and nothing beyond a row is read or written"""
    g = gen(cols)
    rows = 37
    big = [torch.full((rows, cols + 7), math.nan, device="cuda", dtype=dtype) for _ in range(4)]
    x, res, dy, dh = (m[:, 3:3 + cols] for m in big)
    for m in (x, res, dy, dh):
        m.copy_(normal(g, rows, cols))
    w, b = normal(g, cols + 1, to=dtype)[1:], normal(g, cols + 1, to=dtype)[1:]
    got = ops.layernorm_fwd(x, w, b, residual=res)
    compare(got, R.layernorm_fwd(x, w, b, res, 1e-5))
    _, h, mean, rstd = got
    compare(ops.layernorm_bwd(dy, h, w, mean, rstd, dh=dh), R.layernorm_bwd(dy, h, w, mean, rstd, dh))


def test_layernorm_special_values(ops):
    g = gen(6)
    w = torch.ones(256, device="cuda")
    x = normal(g, 4, 256)
    x[1] = 1e4 + x[1] * 1e-2            # a mean far from the spread
    x[2] = 3.0                          # no spread at all
    x[3, 7] = math.nan
    y, _, mean, rstd = ops.layernorm_fwd(x, w)
    compare((y[:3], x[:3], mean[:3], rstd[:3]), R.layernorm_fwd(x[:3], w, None, None, 1e-5))
    assert torch.isnan(y[3]).all()
    assert [t.shape for t in ops.layernorm_fwd(x[:0], w)] == [(0, 256), (0, 256), (0,), (0,)]
    dx, dw, db = ops.layernorm_bwd(x[:0], x[:0], w, mean[:0], rstd[:0])
    assert dx.shape == (0, 256) and not dw.any() and not db.any()


# ---- attention -------------------------------------------------------------------------

def heads(g, B, H, S, D, dtype, layout, scale=1.0):
    if layout == "bshd":
        return normal(g, B, S, H, D, to=dtype, scale=scale).transpose(1, 2)
    if layout == "odd":             # strides that the kernels cannot take as they are
        return normal(g, B, H, S, D + 3, to=dtype, scale=scale)[..., 1:D + 1]
    return normal(g, B, H, S, D, to=dtype, scale=scale)


def some_lengths(g, B, most):
    n = torch.randint(0, most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[0] = most
    if B > 1:
        n[1] = 0
    if B > 2:
        n[2] = 1
    return n


#       B  H  K  Sq    Sk    D   causal ragged layout
ATT = [(1, 1, 1, 1, 1, 64, False, False, "bhsd"),
       (1, 1, 1, 1, 1, 8, True, False, "bhsd"),
       (2, 4, 2, 1, 515, 128, False, False, "bshd"),
       (4, 8, 2, 1, 1200, 128, True, True, "bshd"),
       (1, 8, 1, 3, 1000, 128, False, False, "bhsd"),
       (4, 6, 2, 40, 40, 64, False, True, "bhsd"),
       (4, 6, 2, 40, 40, 64, True, True, "bshd"),
       (1, 2, 2, 129, 65, 80, True, False, "bhsd"),       # 64 queries see nothing
       (1, 2, 1, 65, 257, 128, True, False, "bshd"),
       (2, 4, 4, 200, 200, 32, True, False, "bhsd"),
       (3, 3, 3, 64, 64, 128, False, True, "odd"),
       (1, 16, 2, 31, 2049, 128, True, False, "bhsd"),
       (2, 5, 1, 77, 190, 96, False, True, "bshd"),
       (1, 3, 1, 300, 33, 104, False, False, "bhsd"),
       (1, 1, 1, 700, 700, 16, True, False, "bhsd"),
       (1, 4, 1, 513, 640, 64, True, False, "bshd"),
       (1, 24, 8, 64, 1, 64, True, False, "bhsd"),
       (16, 64, 8, 512, 100, 16, False, False, "bhsd"),    # more than half of the compute units have a block, and long ones: split over queries,
       (1, 8, 8, 2048, 4096, 16, True, False, "bhsd")]     # and over keys


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("case", ATT, ids=lambda c: "-".join(str(x) for x in c))
def test_attention(ops, case, dtype):
    B, H, K, Sq, Sk, D, causal, ragged, layout = case
    g = gen(B * 1000 + Sq * 10 + Sk)
    q, k, v = heads(g, B, H, Sq, D, dtype, layout, 1.5), heads(g, B, K, Sk, D, dtype, layout), heads(g, B, K, Sk, D, dtype, layout)
    dout = heads(g, B, H, Sq, D, dtype, layout)
    more = {"causal": causal}
    if ragged:
        more.update(q_lengths=some_lengths(g, B, Sq) if Sq > 1 else None, kv_lengths=some_lengths(g, B, Sk).flip(0))
    compare(ops.attention_fwd(q, k, v, **more), R.attention_fwd(q, k, v, **more))
    want, o, lse = R.attention_bwd(dout, q, k, v, **more)
    args = dout, q, k, v, o.to(dtype), lse.float()
    first = ops.attention_bwd(*args, **more)
    compare(first, want)
    for a, b in zip(first, ops.attention_bwd(*args, **more)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_does_not_read_what_is_masked(ops, dtype):
    """NaN and infinities beyond the lengths change nothing, and queries without keys give zeros"""
    g = gen(11)
    B, H, K, Sq, Sk, D = 4, 4, 2, 70, 150, 64
    q, k, v, dout = normal(g, B, H, Sq, D, to=dtype), normal(g, B, K, Sk, D, to=dtype), normal(g, B, K, Sk, D, to=dtype), normal(g, B, H, Sq, D, to=dtype)
    nq, nk = torch.tensor([70, 33, 0, 5], dtype=torch.int32, device="cuda"), torch.tensor([150, 0, 77, 65], dtype=torch.int32, device="cuda")
    for causal in (False, True):
        more = {"causal": causal, "q_lengths": nq, "kv_lengths": nk}
        clean = ops.attention_fwd(q, k, v, **more)
        back = ops.attention_bwd(dout, q, k, v, *clean, **more)
        q2, k2, v2, do2, o2 = (t.clone() for t in (q, k, v, dout, clean[0]))
        for b in range(B):
            for t, n in ((q2, nq), (do2, nq), (o2, nq), (k2, nk), (v2, nk)):
                rest = t[b, :, int(n[b]):]
                rest[..., 0::2], rest[..., 1::2] = math.nan, math.inf
        dirty = ops.attention_fwd(q2, k2, v2, **more)
        for a, b in zip(clean, dirty):
            assert torch.equal(a, b)
        for a, b in zip(back, ops.attention_bwd(do2, q2, k2, v2, o2, clean[1], **more)):
            assert torch.equal(a, b)
        assert not clean[0][1].any() and (clean[1][1] == -math.inf).all() and not any(x[1].any() for x in back)


def test_attention_extreme_scores(ops):
    """scores far apart: maxima that move by hundreds between tiles, and the lowest values of the type"""
    g = gen(12)
    q, k, v = normal(g, 1, 2, 40, 64, to=BF16, scale=20), normal(g, 1, 2, 400, 64, to=BF16, scale=8), normal(g, 1, 2, 400, 64, to=BF16)
    k[:, :, 300:] *= 4
    compare(ops.attention_fwd(q, k, v), R.attention_fwd(q, k, v))
    k[0, 0, 5] = torch.finfo(BF16).min / 1e6
    q[0, 0, 3] = 0
    q[0, 0, 4] = 1
    o, lse = ops.attention_fwd(q[:, :, 3:5], k, v, scale=2.0)
    want = R.attention_fwd(q[:, :, 3:5], k, v, scale=2.0)
    R.close(o, *want["o"], "o")
    R.close(lse, *want["lse"], "lse")


def test_attention_small_gradients_in_16_bits(ops):
    """gradients of 1e-4 leave a 16-bit float's exponents when they meet probabilities: they are kept relative to the largest"""
    g = gen(13)
    q, k, v = (normal(g, 1, 2, 600, 64, to=F16) for _ in range(3))
    dout = normal(g, 1, 2, 600, 64, to=F16, scale=2.0 ** -10)
    want, o, lse = R.attention_bwd(dout, q, k, v)
    compare(ops.attention_bwd(dout, q, k, v, o.to(F16), lse.float()), want)
    small = ops.attention_bwd(dout, q, k, v, o.to(F16), lse.float())
    large = ops.attention_bwd(dout * 1024, q, k, v, o.to(F16), lse.float())
    for a, b in zip(small, large):
        # the same products, rounded once to the steps of either size
        R.close(a, b.double() / 1024, R.half(F16) * b.double().abs() / 1024 + R.tiny(F16), "small against large")


def test_attention_no_keys_no_queries(ops):
    q, k = torch.ones(2, 4, 5, 64, dtype=BF16, device="cuda"), torch.ones(2, 2, 0, 64, dtype=BF16, device="cuda")
    o, lse = ops.attention_fwd(q, k, k)
    assert not o.any() and (lse == -math.inf).all()
    dq, dk, dv = ops.attention_bwd(q, q, k, k, o, lse)
    assert not dq.any() and dk.shape == k.shape
    o, lse = ops.attention_fwd(q[:, :, :0], q[:, :2], q[:, :2])
    assert o.shape == (2, 4, 0, 64)
    dq, dk, dv = ops.attention_bwd(o, q[:, :, :0], q[:, :2], q[:, :2], o, lse)
    assert not dk.any() and not dv.any() and dk.shape == (2, 2, 5, 64)
    assert ops.attention_fwd(q[:0], k[:0], k[:0])[0].shape == (0, 4, 5, 64)


def test_attention_gradients_against_differences(ops):
    """loss = <o, dout>: its change along a direction, from two forward passes in 64 bits, against the gradients"""
    g = gen(14)
    q, k, v, dout = (normal(g, 1, 2, 48, 64, to=F16) for _ in range(4))
    o, lse = ops.attention_fwd(q, k, v, causal=True)
    grads = ops.attention_bwd(dout, q, k, v, o, lse, causal=True)
    for n, grad in enumerate(grads):
        d = normal(g, 1, 2, 48, 64).double()
        step, at = 1e-4, [t.double() for t in (q, k, v)]
        loss = []
        for sign in (1, -1):
            moved = list(at)
            moved[n] = at[n] + sign * step * d
            value = R.attention_fwd(*(m.to(torch.float64) for m in moved), causal=True)["o"][0]
            loss.append((value * dout.double()).sum())
        slope = (loss[0] - loss[1]) / (2 * step)
        # each of the 6144 values is off by about 2^-11 of its size at random; six deviations, and the third derivative
        spread = (grad.double() * d).norm() * 2 * 2.0 ** -11 * 6
        assert abs(slope - (grad.double() * d).sum()) < spread + 1e-5 * d.norm(), (n, slope.item())


def of_exact_delta(want, dout, q, k, v, causal):
    """the bounds without the rounding of o: what is left if the row sums of p dp stand for <do, o>"""
    t = q.dtype
    qd, kd, vd, do = (x.double() for x in (q, k, v, dout))
    z = q.shape[3] ** -0.5 * qd @ kd.transpose(2, 3)
    if causal:
        z = z.masked_fill(~R.sees(1, q.shape[2], k.shape[2], True, None, None, q.device), -math.inf)
    p = torch.softmax(z, 3)
    extra = 1.01 * q.shape[3] ** -0.5 * p * R.half(t) * (do * (p @ vd)).abs().sum(3, keepdim=True)
    return {"dq": (want["dq"][0], want["dq"][1] - extra @ kd.abs()), "dk": (want["dk"][0], want["dk"][1] - extra.transpose(2, 3) @ qd.abs())}


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("S,D,causal", [(3, 64, True), (8, 128, True), (40, 64, False), (64, 32, True), (100, 128, False), (128, 64, True)])
def test_attention_rounding_of_o_is_not_in_short_rows(ops, S, D, causal, dtype):
    g = gen(900 + S)
    q, k, v, dout = normal(g, 2, 3, S, D, to=dtype, scale=1.5), *(normal(g, 2, 3, S, D, to=dtype) for _ in range(3))
    want, o, lse = R.attention_bwd(dout, q, k, v, causal=causal)
    dq, dk, _ = ops.attention_bwd(dout, q, k, v, o.to(dtype), lse.float(), causal=causal)
    tight = of_exact_delta(want, dout, q, k, v, causal)
    R.close(dq, *tight["dq"], "dq")
    R.close(dk, *tight["dk"], "dk")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_gradients_of_few_keys_in_the_mean(ops, dtype):
    """dq and dk pass two roundings, of ds and of themselves: each 0.42 of half a step in the mean square where values spread evenly between powers of two,
    0.6 together; with the rounding of o in the row sums they would be off by 0.9 (8 causal keys)"""
    g = gen(980)
    q, k, v, dout = normal(g, 4, 64, 8, 64, to=dtype, scale=1.5), *(normal(g, 4, 64, 8, 64, to=dtype) for _ in range(3))
    want, o, lse = R.attention_bwd(dout, q, k, v, causal=True)
    for name, got in zip(("dq", "dk"), ops.attention_bwd(dout, q, k, v, o.to(dtype), lse.float(), causal=True)):
        assert (got.double() - want[name][0]).norm() < 0.75 * R.half(dtype) * want[name][0].norm(), name


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("cut", [1, 40, 64, 128, 200])
def test_attention_backward_of_keys_in_pieces(ops, cut, dtype):
    """o and lse are those of all keys: each piece gives its own dk and dv, and a part of dq"""
    g = gen(950 + cut)
    q, k, v, dout = normal(g, 1, 4, 90, 64, to=dtype), normal(g, 1, 2, 260, 64, to=dtype), normal(g, 1, 2, 260, 64, to=dtype), normal(g, 1, 4, 90, 64, to=dtype)
    want, o, lse = R.attention_bwd(dout, q, k, v)
    parts = [ops.attention_bwd(dout, q, k[:, :, a:b], v[:, :, a:b], o.to(dtype), lse.float()) for a, b in ((0, cut), (cut, 260))]
    dq = parts[0][0].double() + parts[1][0].double()
    bound = want["dq"][1] + R.half(dtype) * sum(p[0].double().abs() for p in parts) + R.tiny(dtype)
    R.close(dq, want["dq"][0], bound, "dq")
    R.close(torch.cat([p[1] for p in parts], 2), *want["dk"], "dk")
    R.close(torch.cat([p[2] for p in parts], 2), *want["dv"], "dv")


# ---- loss over a vocabulary ------------------------------------------------------------

VOC = [(1, 1, 8), (1, 2, 1), (3, 65, 7), (64, 1000, 64), (65, 129, 72), (130, 515, 100), (257, 700, 33), (5, 33000, 40), (300, 3001, 520), (1200, 900, 128), (70, 64, 1001)]


def vocab_case(g, rows, vocab, dim, dtype, ignored):
    x, w = normal(g, rows, dim, to=dtype), normal(g, vocab, dim, to=dtype, scale=2 / math.sqrt(dim))
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    if ignored:
        t[torch.rand(rows, generator=g, device="cuda") < ignored] = -100
    return x, w, t


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,dim", VOC)
def test_vocab_loss(ops, dtype, rows, vocab, dim):
    g = gen(rows + vocab + dim)
    for ignored in (0.0, 0.3):
        x, w, t = vocab_case(g, rows, vocab, dim, dtype, ignored)
        got = ops.vocab_loss_fwd(x, w, t)
        compare(got, R.vocab_loss_fwd(x, w, t))
        dloss = torch.rand(rows, generator=g, device="cuda") / rows
        first = ops.vocab_loss_bwd(dloss, x, w, t, got[1])
        compare(first, R.vocab_loss_bwd(dloss, x, w, t, got[1]))
        for a, b in zip(first, ops.vocab_loss_bwd(dloss, x, w, t, got[1])):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,rows,vocab,dim", [(BF16, 4100, 4300, 264), (F16, 4096, 33000, 72)])
def test_vocab_loss_of_large_tiles_and_pieces(ops, dtype, rows, vocab, dim):
    """enough rows and words for the large tiles; and more of both than one piece's gradient of the logits holds"""
    g = gen(vocab)
    x, w, t = vocab_case(g, rows, vocab, dim, dtype, 0.1)
    got = ops.vocab_loss_fwd(x, w, t)
    compare(got, R.vocab_loss_fwd(x, w, t))
    dloss = torch.full((rows,), 1.0 / rows, device="cuda")
    compare(ops.vocab_loss_bwd(dloss, x, w, t, got[1]), R.vocab_loss_bwd(dloss, x, w, t, got[1]))


def test_vocab_loss_in_shards(ops):
    """two devices' shares of the vocabulary: joined statistics give the whole loss, the shares of dx add up"""
    g = gen(21)
    x, w, t = vocab_case(g, 90, 700, 96, BF16, 0.2)
    cut = 263
    parts = [ops.vocab_loss_fwd(x, w[a:b], t, first_word=a) for a, b in ((0, cut), (cut, 700))]
    assert parts[0][0] is None
    for (a, b), p in zip(((0, cut), (cut, 700)), parts):
        want = R.vocab_loss_fwd(x, w[a:b], t, first=a)
        R.close(p[1], *want["lse"], "lse")
        R.close(p[2], *want["target_logit"], "target_logit")
    lse = torch.logsumexp(torch.stack([p[1] for p in parts]), 0)
    whole = R.vocab_loss_fwd(x, w, t)
    loss = torch.where(t == -100, 0.0, lse - parts[0][2] - parts[1][2])
    R.close(loss, whole["loss"][0], whole["loss"][1] * 2, "loss")
    dloss = torch.rand(90, generator=g, device="cuda")
    for a, b in ((0, cut), (cut, 700)):
        compare(ops.vocab_loss_bwd(dloss, x, w[a:b], t, lse, first_word=a), R.vocab_loss_bwd(dloss, x, w[a:b], t, lse, first=a))


def test_vocab_loss_targets_and_strides(ops):
    g = gen(22)
    x, w, t = vocab_case(g, 70, 300, 64, BF16, 0.0)
    t[3], t[4], t[5], t[6] = 300, -1, -100, 2 ** 31 - 1
    got = ops.vocab_loss_fwd(x, w, t)
    compare(got, R.vocab_loss_fwd(x, w, t))
    assert torch.isnan(got[0][[3, 4, 6]]).all() and got[0][5] == 0
    dloss = torch.ones(70, device="cuda")
    dx, dw = ops.vocab_loss_bwd(dloss, x, w, t, got[1])
    compare((dx, dw), R.vocab_loss_bwd(dloss, x, w, t, got[1]))
    assert not dx[5].any()
    t[:] = 7
    got = ops.vocab_loss_fwd(x, w, t, ignore_index=7)
    assert not got[0].any() and not any(y.any() for y in ops.vocab_loss_bwd(dloss, x, w, t, got[1], ignore_index=7))
    # slices of wider matrices, repeated rows, columns first
    big = normal(g, 70, 200, to=BF16)
    for xs, ws in ((big[:, 8:72], w), (big[:, 3:67], w), (big[:1, :64].expand(70, 64), w), (x, normal(g, 64, 300, to=BF16).t()), (x, normal(g, 300, 70, to=BF16)[:, 5:69])):
        t = torch.randint(0, 300, (70,), generator=g, device="cuda", dtype=torch.int32)
        got = ops.vocab_loss_fwd(xs, ws, t)
        compare(got, R.vocab_loss_fwd(xs, ws, t))
        compare(ops.vocab_loss_bwd(dloss, xs, ws, t, got[1]), R.vocab_loss_bwd(dloss, xs, ws, t, got[1]))
    loss, lse, _ = ops.vocab_loss_fwd(x[:0], w, t[:0])
    assert loss.shape == (0,)
    dx, dw = ops.vocab_loss_bwd(dloss[:0], x[:0], w, t[:0], lse)
    assert dx.shape == (0, 64) and dw.shape == w.shape and not dw.any()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,dim", [(5, 70, 33), (64, 300, 64), (65, 515, 100), (700, 1300, 72), (2100, 600, 64), (9000, 130, 16)])
@pytest.mark.parametrize("share", [0.03, 0.5, 0.97, 1.0])
def test_vocab_loss_rows_that_take_no_part(ops, rows, vocab, dim, share, dtype):
    """their vectors, weights and statistics may hold anything, and the others' gradients are those of a call without them"""
    g = gen(rows + int(share * 100))
    x, w, t = vocab_case(g, rows, vocab, dim, dtype, 0.0)
    dloss = normal(g, rows)
    out = torch.rand(rows, generator=g, device="cuda") < share
    t[out] = -100
    x[out] = math.nan
    dloss[out] = math.inf
    _, lse, _ = ops.vocab_loss_fwd(x, w, t)
    dx, dw = ops.vocab_loss_bwd(dloss, x, w, t, lse)
    assert not dx[out].any()
    some = R.vocab_loss_bwd(dloss[~out], x[~out], w, t[~out], lse[~out])
    R.close(dx[~out], *some["dx"], "dx")
    R.close(dw, *some["dw"], "dw")


def test_vocab_loss_large_logits(ops):
    """logits of hundreds, all of them negative for some rows"""
    g = gen(23)
    x, w, t = vocab_case(g, 64, 500, 64, BF16, 0.0)
    x, w = x * 10, w.abs() * 4
    x[5] = -x[5].abs() * 4
    got = ops.vocab_loss_fwd(x, w, t)
    compare(got, R.vocab_loss_fwd(x, w, t))
    dloss = torch.ones(64, device="cuda")
    compare(ops.vocab_loss_bwd(dloss, x, w, t, got[1]), R.vocab_loss_bwd(dloss, x, w, t, got[1]))


# ---- streams and graphs ----------------------------------------------------------------

def test_operators_on_another_stream_and_in_a_graph(ops):
    """the same bits on a side stream and in three replays of a captured graph with new inputs and eager work between them"""
    g = gen(31)
    x, w, b = normal(g, 200, 256, to=F16), normal(g, 256, to=F16), normal(g, 256, to=F16)
    q, k, v, dout = (normal(g, 2, 4, 90, 64, to=F16) for _ in range(4))
    voc, t = normal(g, 999, 256, to=F16, scale=0.1), torch.randint(0, 999, (200,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.full((200,), 0.005, device="cuda")

    def everything():
        y, h, mean, rstd = ops.layernorm_fwd(x, w, b)
        loss, lse, _ = ops.vocab_loss_fwd(y, voc, t)
        dy, dvoc = ops.vocab_loss_bwd(dloss, y, voc, t, lse)
        dx, dw, db = ops.layernorm_bwd(dy, h, w, mean, rstd)
        o, l = ops.attention_fwd(q, k, v, causal=True)
        return [y, loss, dvoc, dx, dw, db, o, *ops.attention_bwd(dout, q, k, v, o, l, causal=True)]

    want = [r.clone() for r in everything()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = everything()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for n in range(3):
        x.add_(0.25)
        q.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = everything()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out)), n

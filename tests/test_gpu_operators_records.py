"""What include/ff_ops.h allows beyond the functions on tensors: outputs in the memory of inputs, outputs that are not asked for."""
import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import operators as O  # noqa: E402

pytestmark = pytest.mark.gpu

CODES = {torch.float32: O.FF_F32, torch.float16: O.FF_F16, torch.bfloat16: O.FF_BF16}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, to):
    return torch.randn(*shape, generator=g, device="cuda").to(to)


def copy_of(t):
    """with the strides and the alignment of t, as which results may differ in the last bit"""
    big = torch.empty(t.shape[0] * t.stride(0) + 64, device="cuda", dtype=t.dtype)
    at = t.data_ptr() // t.element_size() % 64
    return big[at:].as_strided(t.shape, t.stride()).copy_(t)


def rows_of(t):
    return O.ff_rows_t(None if t is None else t.data_ptr(), 0 if t is None else t.stride(0))


def launch(name, record):
    if name + "_workspace_bytes" in O.EXPORTS:
        n = O.workspace_bytes(name, record)
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
        record.workspace, record.workspace_bytes = ws.data_ptr(), n
    O.call(name, record, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,wide", [(5, 7, 9), (37, 64, 64), (19, 100, 103), (40, 1000, 1000), (33, 2047, 2050), (21, 5000, 5001), (7, 9001, 9001), (5, 20000, 20000)])
def test_layernorm_in_place(dtype, rows, cols, wide):
    g = gen(cols)
    x, res, dy, dh = (normal(g, rows, wide, to=dtype)[:, wide - cols:] for _ in range(4))
    w, b = normal(g, cols, to=dtype), normal(g, cols, to=dtype)
    y, h, mean, rstd = O.layernorm_fwd(x, w, b, residual=res)
    dx, dw, db = O.layernorm_bwd(dy, h, w, mean, rstd, dh=dh)
    for into in (0, 1):         # y in the memory of x, and of res
        a, r, hh = copy_of(x), copy_of(res), torch.empty_like(h)
        launch("ff_op_layernorm_fwd", O.ff_layernorm_fwd_t(CODES[dtype], cols, rows, 1e-5, rows_of(a), rows_of(r), rows_of(hh), rows_of((a, r)[into]), w.data_ptr(), b.data_ptr(), None, None))
        assert torch.equal((a, r)[into], y) and torch.equal(hh, h)
        a, r = copy_of(dy), copy_of(dh)   # dx in the memory of dy, and of dh, with one gradient of the weights at a time
        gw = torch.full_like(dw, 7)
        rec = O.ff_layernorm_bwd_t(CODES[dtype], cols, rows, rows_of(a), rows_of(h), rows_of(r), rows_of((a, r)[into]), w.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                   None if into else gw.data_ptr(), gw.data_ptr() if into else None, None, 0)
        launch("ff_op_layernorm_bwd", rec)
        assert torch.equal((a, r)[into], dx) and torch.equal(gw, db if into else dw)
    a = copy_of(dy)
    launch("ff_op_layernorm_bwd", O.ff_layernorm_bwd_t(CODES[dtype], cols, rows, rows_of(a), rows_of(h), rows_of(dh), rows_of(a), w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), None, None, None, 0))
    assert torch.equal(a, dx)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,dim", [(50, 70, 33), (300, 3001, 520), (1003, 11003, 1000)])
def test_vocab_loss_outputs_that_are_not_asked_for(dtype, rows, vocab, dim):
    g = gen(vocab)
    x, w = normal(g, rows, dim, to=dtype), (normal(g, vocab, dim, to=torch.float32) / dim ** 0.5).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    t[::5] = -100
    loss, lse, logit = O.vocab_loss_fwd(x, w, t)
    for asked in ((1, 0), (0, 1), (0, 0)):
        a, l, b = (torch.full_like(lse, 7) for _ in range(3))
        rec = O.ff_vocab_loss_fwd_t(CODES[dtype], rows, vocab, dim, -100, 0, rows_of(x), rows_of(w), t.data_ptr(), a.data_ptr() if asked[0] else None, l.data_ptr(), b.data_ptr() if asked[1] else None)
        launch("ff_op_vocab_loss_fwd", rec)
        assert torch.equal(l, lse) and torch.equal(a, loss if asked[0] else torch.full_like(a, 7)) and torch.equal(b, logit if asked[1] else torch.full_like(b, 7))
    dloss = torch.rand(rows, generator=g, device="cuda")
    dx, dw = O.vocab_loss_bwd(dloss, x, w, t, lse)
    for n in (0, 1):
        out = torch.full_like((dx, dw)[n], 7)
        rec = O.ff_vocab_loss_bwd_t(CODES[dtype], rows, vocab, dim, -100, 0, rows_of(x), rows_of(w), rows_of(None if n else out), rows_of(out if n else None), t.data_ptr(), dloss.data_ptr(), lse.data_ptr())
        launch("ff_op_vocab_loss_bwd", rec)
        assert torch.equal(out, (dx, dw)[n])


@pytest.mark.parametrize("rows,dim", [(70, 33), (300, 520)])
def test_vocab_loss_outputs_in_wider_rows(rows, dim):
    """rows of dx and dw that lie apart, at any place: nothing beside them is written"""
    g = gen(dim)
    dtype, vocab = torch.bfloat16, 515
    x, w = normal(g, rows, dim, to=dtype), (normal(g, vocab, dim, to=torch.float32) / dim ** 0.5).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    _, lse, _ = O.vocab_loss_fwd(x, w, t)
    dloss = torch.rand(rows, generator=g, device="cuda")
    dx, dw = O.vocab_loss_bwd(dloss, x, w, t, lse)
    for at, wide in ((1, dim + 3), (3, dim + 8), (8, dim + 16)):
        bx, bw = torch.full((rows, wide), 7.0, device="cuda", dtype=dtype), torch.full((vocab, wide), 7.0, device="cuda", dtype=dtype)
        ox, ow = bx[:, at:at + dim], bw[:, at:at + dim]
        launch("ff_op_vocab_loss_bwd", O.ff_vocab_loss_bwd_t(CODES[dtype], rows, vocab, dim, -100, 0, rows_of(x), rows_of(w), rows_of(ox), rows_of(ow), t.data_ptr(), dloss.data_ptr(), lse.data_ptr()))
        assert torch.equal(ox, dx) and torch.equal(ow, dw)
        for big in (bx, bw):
            assert (big[:, :at] == 7).all() and (big[:, at + dim:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Sq,Sk,D", [(40, 40, 64), (130, 300, 80), (1, 5000, 128)])
def test_attention_outputs_in_wider_heads(Sq, Sk, D, dtype):
    """heads of outputs that lie apart, positions outside: nothing beside them is written"""
    g = gen(Sq + Sk)
    B, H, K = 2, 4, 2
    q, dout = normal(g, B, H, Sq, D, to=dtype), normal(g, B, H, Sq, D, to=dtype)
    k, v = normal(g, B, K, Sk, D, to=dtype), normal(g, B, K, Sk, D, to=dtype)
    o, lse = O.attention_fwd(q, k, v, causal=True)
    grads = O.attention_bwd(dout, q, k, v, o, lse, causal=True)

    def heads(t):
        return O.ff_heads_t(t.data_ptr(), *t.stride()[:3])

    def apart(n, S):
        big = torch.full((B, S, n, D + 16), 7.0, device="cuda", dtype=dtype)
        return big, big[..., 8:8 + D].transpose(1, 2)

    sizes = (CODES[dtype], B, H, K, Sq, Sk, D, 1, D ** -0.5)
    big, out = apart(H, Sq)
    l = torch.empty_like(lse)
    launch("ff_op_attention_fwd", O.ff_attention_fwd_t(*sizes, heads(q), heads(k), heads(v), heads(out), l.data_ptr(), None, None))
    assert torch.equal(out, o) and torch.equal(l, lse) and (big[..., :8] == 7).all() and (big[..., 8 + D:] == 7).all()
    outs = [apart(H, Sq), apart(K, Sk), apart(K, Sk)]
    launch("ff_op_attention_bwd", O.ff_attention_bwd_t(*sizes, heads(dout), heads(q), heads(k), heads(v), heads(o), *(heads(t) for _, t in outs), lse.data_ptr(), None, None))
    for (big, out), want in zip(outs, grads):
        assert torch.equal(out, want) and (big[..., :8] == 7).all() and (big[..., 8 + D:] == 7).all()

"""CPU-side checks of the operators' boundary: exports and record layouts match include/ff_ops.h, malformed records are refused
before anything is launched, and the functions on top refuse what they cannot take."""
import ctypes as C
import os
import re
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import binding, operators as O  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ff_ops.h")
P = 1 << 20         # an aligned address that nothing reads: every call below is refused on the host
INVALID, RANGE, WORKSPACE = binding.FF_EINVAL, binding.FF_ERANGE, binding.FF_EWORKSPACE


def test_exports_match_the_header():
    declared = set(re.findall(r"\b(ff_op_\w+)\s*\(", open(HEADER).read()))
    assert declared == set(O.EXPORTS)
    for name in declared:
        assert hasattr(O.lib(), name), name


def test_record_layouts_match_the_header(tmp_path):
    """size and place of every field, as a C compiler sees them"""
    records = [O.ff_rows_t, O.ff_heads_t, *O._RECORDS.values()]
    lines = [f'printf("{r.__name__}.{f[0]} %zu\\n", offsetof({r.__name__}, {f[0]}));' for r in records for f in r._fields_]
    lines += [f'printf("{r.__name__} %zu\\n", sizeof({r.__name__}));' for r in records]
    src = tmp_path / "layout.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void) {{\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-o", str(tmp_path / "layout"), str(src)])
    said = dict(line.rsplit(" ", 1) for line in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines())
    for r in records:
        assert int(said[r.__name__]) == C.sizeof(r)
        for f in r._fields_:
            assert int(said[f"{r.__name__}.{f[0]}"]) == getattr(r, f[0]).offset, f[0]


def put(rec, **fields):
    for k, v in fields.items():
        *path, last = k.split("__")
        at = rec
        for p in path:
            at = getattr(at, p)
        setattr(at, last, v)
    return rec


def code(name, rec):
    return getattr(O.lib(), name)(C.byref(rec), None)


def good_layernorm_fwd():
    r = O.ff_rows_t(P, 64)
    return O.ff_layernorm_fwd_t(O.FF_BF16, 64, 4, 1e-5, r, O.ff_rows_t(None, 0), O.ff_rows_t(None, 0), r, P, P, P, P)


def good_layernorm_bwd():
    r = O.ff_rows_t(P, 64)
    return O.ff_layernorm_bwd_t(O.FF_BF16, 64, 4, r, r, O.ff_rows_t(None, 0), r, P, P, P, P, P, P, 1 << 30)


def good_attention(cls, names):
    h = O.ff_heads_t(P, 8 * 16 * 64, 16 * 64, 64)
    rec = cls(O.FF_F16, 2, 8, 2, 16, 16, 64, 0, 0.125)
    for n in names:
        setattr(rec, n, h)
    return put(rec, lse=P, workspace=P, workspace_bytes=1 << 30)


def good_vocab(cls, **fields):
    r = O.ff_rows_t(P, 64)
    return put(cls(O.FF_BF16, 4, 100, 64, -100, 0, r, r), targets=P, lse=P, workspace=P, workspace_bytes=1 << 30, **fields)


GOOD = {"ff_op_layernorm_fwd": good_layernorm_fwd, "ff_op_layernorm_bwd": good_layernorm_bwd,
        "ff_op_attention_fwd": lambda: good_attention(O.ff_attention_fwd_t, "qkvo"),
        "ff_op_attention_bwd": lambda: good_attention(O.ff_attention_bwd_t, ("dout", "q", "k", "v", "o", "dq", "dk", "dv")),
        "ff_op_vocab_loss_fwd": lambda: good_vocab(O.ff_vocab_loss_fwd_t),
        "ff_op_vocab_loss_bwd": lambda: good_vocab(O.ff_vocab_loss_bwd_t, dloss=P, dx=O.ff_rows_t(P, 64), dw=O.ff_rows_t(P, 64))}

NAN, INF = float("nan"), float("inf")
BAD = {
    "ff_op_layernorm_fwd": [(INVALID, dict(dtype=3)), (INVALID, dict(cols=0)), (RANGE, dict(cols=65537)), (RANGE, dict(rows=1 << 29)), (INVALID, dict(eps=NAN)), (INVALID, dict(eps=-1.0)),
                            (INVALID, dict(eps=INF)), (INVALID, dict(x__p=None)), (INVALID, dict(y__p=None)), (INVALID, dict(weight=None)), (INVALID, dict(res=O.ff_rows_t(P, 64)))],
    "ff_op_layernorm_bwd": [(INVALID, dict(dtype=7)), (INVALID, dict(cols=0)), (RANGE, dict(cols=1 << 20)), (RANGE, dict(rows=1 << 40)), (INVALID, dict(dy__p=None)), (INVALID, dict(h__p=None)),
                            (INVALID, dict(dx__p=None)), (INVALID, dict(weight=None)), (INVALID, dict(mean=None)), (INVALID, dict(rstd=None)), (WORKSPACE, dict(workspace=None)),
                            (WORKSPACE, dict(workspace_bytes=511)), (WORKSPACE, dict(workspace=P + 16))],
    "ff_op_attention_fwd": [(INVALID, dict(dtype=O.FF_F32)), (INVALID, dict(kv_heads=0)), (INVALID, dict(heads=0)), (INVALID, dict(heads=7)), (INVALID, dict(head_dim=0)), (INVALID, dict(head_dim=60)),
                            (RANGE, dict(head_dim=136)), (RANGE, dict(kv_len=(1 << 28) + 1)), (RANGE, dict(q_len=1 << 28)), (RANGE, dict(batch=65536)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=NAN)),
                            (INVALID, dict(scale=INF)), (INVALID, dict(q__p=None)), (INVALID, dict(k__p=None)), (INVALID, dict(v__p=P + 2)), (INVALID, dict(o__p=P + 8)), (INVALID, dict(q__pos=63)),
                            (INVALID, dict(k__head=4)), (INVALID, dict(v__batch=12)), (INVALID, dict(lse=None)), (WORKSPACE, dict(batch=1, kv_len=4096, workspace=None)),
                            (WORKSPACE, dict(batch=1, kv_len=4096, workspace_bytes=100)), (WORKSPACE, dict(batch=1, kv_len=4096, workspace=P + 128))],
    "ff_op_attention_bwd": [(INVALID, dict(dtype=O.FF_F32)), (INVALID, dict(heads=3)), (INVALID, dict(head_dim=12)), (RANGE, dict(head_dim=256)), (INVALID, dict(scale=0.0)), (INVALID, dict(lse=None))] +
                           [(INVALID, {n + "__p": None}) for n in ("dout", "q", "k", "v", "o", "dq", "dk", "dv")] + [(INVALID, {n + "__pos": 20}) for n in ("dout", "q", "k", "v", "o", "dq", "dk", "dv")] +
                           [(WORKSPACE, dict(workspace=None)), (WORKSPACE, dict(workspace_bytes=64)), (WORKSPACE, dict(workspace=P + 4))],
    "ff_op_vocab_loss_fwd": [(INVALID, dict(dtype=O.FF_F32)), (INVALID, dict(vocab=0)), (INVALID, dict(dim=0)), (RANGE, dict(dim=65537)), (RANGE, dict(vocab=1 << 29)), (RANGE, dict(rows=1 << 29)),
                             (RANGE, dict(rows=1 << 28, vocab=1 << 28)), (INVALID, dict(x__p=None)), (INVALID, dict(w__p=None)), (INVALID, dict(targets=None)), (INVALID, dict(lse=None)),
                             (WORKSPACE, dict(workspace=None)), (WORKSPACE, dict(workspace_bytes=16)), (WORKSPACE, dict(workspace=P + 64))],
    "ff_op_vocab_loss_bwd": [(INVALID, dict(dtype=5)), (INVALID, dict(vocab=0)), (INVALID, dict(dim=0)), (RANGE, dict(dim=1 << 17)), (INVALID, dict(x__p=None)), (INVALID, dict(w__p=None)),
                             (INVALID, dict(targets=None)), (INVALID, dict(dloss=None)), (INVALID, dict(lse=None)), (WORKSPACE, dict(workspace=None)), (WORKSPACE, dict(workspace_bytes=256)),
                             (WORKSPACE, dict(workspace=P + 8))],
}


@pytest.mark.parametrize("name", sorted(BAD))
def test_malformed_records_are_refused(name):
    assert getattr(O.lib(), name)(None, None) == INVALID
    for want, fields in BAD[name]:
        rec = put(GOOD[name](), **fields)
        assert code(name, rec) == want, fields
    if name + "_workspace_bytes" in O.EXPORTS:
        size = getattr(O.lib(), name + "_workspace_bytes")
        assert size(None) == 0 and size(C.byref(put(GOOD[name](), dtype=9))) == 0


def test_nothing_to_do_is_fine():
    """no rows, no sequences: FF_OK without a launch"""
    assert code("ff_op_layernorm_fwd", put(good_layernorm_fwd(), rows=0)) == 0
    assert code("ff_op_layernorm_bwd", put(good_layernorm_bwd(), rows=0, dweight=None, dbias=None)) == 0
    for name in ("ff_op_attention_fwd", "ff_op_attention_bwd"):
        assert code(name, put(GOOD[name](), batch=0)) == 0
    assert code("ff_op_vocab_loss_fwd", put(GOOD["ff_op_vocab_loss_fwd"](), rows=0)) == 0
    assert code("ff_op_vocab_loss_bwd", put(GOOD["ff_op_vocab_loss_bwd"](), dx__p=None, dw__p=None)) == 0


def test_workspaces_grow_with_the_sizes_and_stay_bounded():
    size = lambda name, **f: O.workspace_bytes(name, put(GOOD[name](), **f))
    assert size("ff_op_attention_fwd") == 0                                         # nothing is split
    assert size("ff_op_attention_fwd", batch=1, q_len=1, kv_len=100000) > 0
    assert size("ff_op_attention_bwd", q_len=4096) >= 2 * 8 * 4096 * 4
    # the logits of 8192 tokens and 50000 words would be 800 MB in 16 bits: no piece of them takes more than 256 MB
    assert size("ff_op_vocab_loss_bwd", rows=8192, vocab=50000, dim=64) < (256 << 20) + 16 * 8192 * 64 * 4 + 8192 * 16
    assert size("ff_op_vocab_loss_fwd", rows=8192, vocab=50000, dim=64) < 8192 * 4 * (2 * 50000 // 64 + 8)


def test_functions_refuse_what_they_cannot_take():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    q = torch.zeros(2, 4, 8, 64, dtype=torch.float16)
    for bad in (lambda: O.layernorm_fwd(x, w),                                       # not on a GPU
                lambda: O.layernorm_fwd(x[0], w), lambda: O.layernorm_fwd(x.double(), w),
                lambda: O.layernorm_bwd(x, x[0], w, w, w),
                lambda: O.attention_fwd(q, q, q), lambda: O.attention_fwd(q.float(), q.float(), q.float()), lambda: O.attention_fwd(q[0], q, q),
                lambda: O.vocab_loss_fwd(x, x, torch.zeros(4, dtype=torch.int32)), lambda: O.vocab_loss_fwd(x.float(), x.float(), torch.zeros(4, dtype=torch.int32)),
                lambda: O.vocab_loss_bwd(None, x[0], x, None, None)):
        with pytest.raises(ValueError):
            bad()

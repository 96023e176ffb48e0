"""The operators' limits on the host: every launch has fewer than 2^32 threads along x and 2^16 blocks along y, or the record is refused before the first one.
All records lack an address or a workspace, which is asked for after the sizes, so that nothing is launched."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import binding, operators as O  # noqa: E402
from test_operators_refusals import GOOD, code, put  # noqa: E402

INVALID, RANGE, WORKSPACE = binding.FF_EINVAL, binding.FF_ERANGE, binding.FF_EWORKSPACE
SIDE, TOKENS = 65535 * 128, (1 << 26) - 4


@pytest.mark.parametrize("name,want,fields", [
    ("ff_op_layernorm_fwd", INVALID, dict(rows=1 << 28, cols=1024)),
    ("ff_op_layernorm_fwd", RANGE, dict(rows=(1 << 28) + 1, cols=1024)),
    # rows of the queries' side, 4 heads each here
    ("ff_op_attention_fwd", INVALID, dict(q_len=SIDE // 4)),
    ("ff_op_attention_fwd", RANGE, dict(q_len=SIDE // 4 + 1)),
    ("ff_op_attention_fwd", INVALID, dict(kv_len=1 << 28, q_len=1)),
    ("ff_op_attention_bwd", WORKSPACE, dict(q_len=SIDE // 4)),
    ("ff_op_attention_bwd", RANGE, dict(q_len=SIDE // 4 + 1)),
    ("ff_op_attention_bwd", WORKSPACE, dict(kv_len=SIDE)),
    ("ff_op_attention_bwd", RANGE, dict(kv_len=SIDE + 1)),
    ("ff_op_attention_bwd", RANGE, dict(kv_len=1 << 28)),
    ("ff_op_vocab_loss_fwd", WORKSPACE, dict(rows=TOKENS, vocab=64)),
    ("ff_op_vocab_loss_fwd", RANGE, dict(rows=TOKENS + 1, vocab=64)),
    ("ff_op_vocab_loss_fwd", WORKSPACE, dict(vocab=TOKENS, rows=64)),
    ("ff_op_vocab_loss_fwd", RANGE, dict(vocab=TOKENS + 1, rows=64)),
    # 2^11 x 2^13 tiles of 128 x 128 are one too many, 2^12 x 2^12 of 256 x 256 as well
    ("ff_op_vocab_loss_fwd", RANGE, dict(rows=1 << 18, vocab=1 << 20)),
    ("ff_op_vocab_loss_fwd", WORKSPACE, dict(rows=1 << 18, vocab=(1 << 20) - 128)),
    ("ff_op_vocab_loss_fwd", RANGE, dict(rows=1 << 20, vocab=1 << 20, dim=512)),
    ("ff_op_vocab_loss_fwd", WORKSPACE, dict(rows=1 << 20, vocab=(1 << 20) - 256, dim=512)),
    ("ff_op_vocab_loss_bwd", WORKSPACE, dict(rows=TOKENS, vocab=64)),
    ("ff_op_vocab_loss_bwd", RANGE, dict(rows=TOKENS + 1, vocab=64)),
    ("ff_op_vocab_loss_bwd", RANGE, dict(vocab=TOKENS + 1)),
    # rows x dim in tiles of 128 x 128 (few words); dim x words with one row
    ("ff_op_vocab_loss_bwd", RANGE, dict(rows=1 << 22, dim=65536)),
    ("ff_op_vocab_loss_bwd", RANGE, dict(rows=1, vocab=TOKENS, dim=65536)),
    # dx summed over pieces: rows * dim / 4 threads
    ("ff_op_vocab_loss_bwd", RANGE, dict(rows=1 << 21, vocab=1000, dim=8200)),
    ("ff_op_vocab_loss_bwd", WORKSPACE, dict(rows=1 << 21, vocab=1000, dim=8184)),
])
def test_both_sides_of_the_limits(name, want, fields):
    lacking = {"ff_op_layernorm_fwd": dict(x__p=None), "ff_op_attention_fwd": dict(q__p=None)}.get(name, dict(workspace=None))
    assert code(name, put(GOOD[name](), **lacking, **fields)) == want
    if want == RANGE and name + "_workspace_bytes" in O.EXPORTS:
        assert getattr(O.lib(), name + "_workspace_bytes")(C.byref(put(GOOD[name](), **fields))) == 0

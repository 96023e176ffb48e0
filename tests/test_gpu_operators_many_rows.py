"""Layer norm of more rows than one launch takes."""
import pytest

torch = pytest.importorskip("torch")

import operators_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu


def test_layernorm_of_the_most_rows():
    """2^28 rows of 2 elements: 2^24 blocks of 256 threads, one more than a launch may have"""
    from paper_1807_05358_amd import operators as ops
    rows, cols = 1 << 28, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, res = (torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    w, b = (torch.randn(cols, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    got = ops.layernorm_fwd(x, w, b, residual=res)
    for at in (0, rows // 2, rows - 2 ** 12, rows - 64):        # the last block's rows, and others
        part = slice(at, at + 64)
        for (name, (value, bound)), y in zip(R.layernorm_fwd(x[part], w, b, res[part], 1e-5).items(), got):
            R.close(y[part], value, bound, name)
    assert torch.equal(got[1], x + res)
    y, h, mean, rstd = ops.layernorm_fwd(x, w, b)
    part = slice(rows - 64, rows)
    for (name, (value, bound)), z in zip(R.layernorm_fwd(x[part], w, b, None, 1e-5).items(), (y, h, mean, rstd)):
        R.close(z[part], value, bound, name)

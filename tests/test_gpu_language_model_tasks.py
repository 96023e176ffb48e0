"""What the example's measurement runs for a task is the graph's operation, no more and no less."""
import pytest

torch = pytest.importorskip("torch")

from paper_1807_05358_amd import language_model as L, workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_norms_task_has_no_residual_sum(monkeypatch):
    """the graph has the sum as an operation of its own, with a time of its own"""
    asked = []

    def spy(name):
        plain = getattr(L.O, name)

        def call(*args, **more):
            asked.append((name, more.get("residual"), more.get("dh")))
            return plain(*args, **more)
        monkeypatch.setattr(L.O, name, call)

    spy("layernorm_fwd")
    spy("layernorm_bwd")
    measure = L.DeviceMeasure(64, 32, repeats=2)
    for back in (0, L.BACKWARD):
        assert measure(L.T_NORM + back, (2, 8, 64)) > 0
    assert {n for n, _, _ in asked} == {"layernorm_fwd", "layernorm_bwd"}
    assert all(residual is None and dh is None for _, residual, dh in asked)
    ops = L.graph(batch=4, length=32, hidden=64, vocab=512, layers=1)[0]
    assert (ops["type"] == W.T_ELEM).sum() == 2


def test_the_embeddings_table_has_the_words_of_the_vocabulary():
    measure = L.DeviceMeasure(64, 32, vocab=5000)
    grad = measure._task(W.T_EMBED + L.BACKWARD, (2, 8, 16))()
    assert grad.shape == (5000, 16) and grad.dtype == torch.bfloat16
    assert measure._task(W.T_EMBED, (2, 8, 16))().shape == (16, 16)

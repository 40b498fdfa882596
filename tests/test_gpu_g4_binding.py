"""What the binding of the calls on 4-bit weights refuses on a GPU, before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def test_packing_looks_at_the_device(t, qnn, monkeypatch):
    """Weights of another device than the current one are refused, as the rows of the other calls are."""
    w = t.ones((8, 64), device=DEV)
    launched = []
    monkeypatch.setattr(qnn, "_stream", lambda stream=None: launched.append(stream))
    monkeypatch.setattr(qnn.lib, "qnn_g4_pack_weights", lambda *a: launched.append(a) or 0)
    with monkeypatch.context() as m:
        m.setattr(t.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current CUDA device"):
            qnn.g4_pack_weights(w)
    assert not launched
    monkeypatch.undo()
    assert qnn.g4_pack_weights(w).alpha.item() > 0

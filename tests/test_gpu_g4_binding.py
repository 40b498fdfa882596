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


def test_results_that_require_grad_are_refused_and_functions_are_not(t, qnn):
    """Results given by the caller; and the way that stays open: the calls inside an autograd.Function."""
    offsets = t.tensor([0, 5], dtype=t.int32, device=DEV)
    w = qnn.g4_pack_weights(t.randn((24, 40), device=DEV).requires_grad_())
    x = t.randn((5, 40), device=DEV)
    dy = t.randn((5, 24), device=DEV)
    with pytest.raises(ValueError, match="record no gradients"):
        qnn.g4_expert_gemm(x, w, offsets, out=t.zeros((5, 24), device=DEV, requires_grad=True))
    with pytest.raises(ValueError, match="record no gradients"):
        qnn.expert_gemm_backward_weights(dy, x, offsets, gw=t.zeros((1, 24, 40), device=DEV, requires_grad=True))

    class Product(t.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return qnn.g4_expert_gemm(x, w, offsets)

        @staticmethod
        def backward(ctx, dy):
            return qnn.g4_expert_gemm_backward_data(dy.contiguous(), w, offsets)
    xg = x.clone().requires_grad_()
    (Product.apply(xg) * dy).sum().backward()
    assert t.equal(xg.grad, qnn.g4_expert_gemm_backward_data(dy, w, offsets))


def test_experts_layer_repeats_its_bits(t, qnn):
    """Four experts a token: their results are added in a fixed order, so the layer of run_case gives the same bits every time."""
    from paper_2106_09886_b200.run_case import ExpertsLayer
    layer = ExpertsLayer(256, 384, 8, 4, 64, group=64, dtype=t.float32, seed=5)
    x = t.randn((700, 256), device=DEV, generator=t.Generator(device=DEV).manual_seed(6))
    first = layer.forward(x)[0]
    for _ in range(20):
        assert t.equal(layer.forward(x)[0], first)

"""Operands that carry a forward-mode tangent are refused by the calls of the compiled module, which would drop it: on the host, before
anything else about the operands is asked."""
import pytest


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import build
    build.build()
    from paper_2106_09886_b200 import qnn as q
    return q


def calls(t, qnn, dual):
    """name -> a call whose one operand carries a tangent"""
    x, v, ints = t.randn(4, 32), t.randn(32), t.zeros((4, 2), dtype=t.int32)
    rstd, scales, codes = t.ones(4), t.ones(4), t.zeros((4, 32), dtype=t.int8)
    rows = qnn.I8Rows(codes, scales)
    weights = qnn.G4Weights(t.zeros((2, 1, 1, 4, 128, 4), dtype=t.int32), t.zeros((2, 1, 1, 4, 128), dtype=t.uint8), t.ones(2), 32, 32, 32)
    offsets = t.tensor([0, 2, 4], dtype=t.int32)
    return {
        "rms_norm x": lambda: qnn.rms_norm(dual(x), v), "rms_norm gain": lambda: qnn.rms_norm(x, dual(v)),
        "rms_norm residual": lambda: qnn.rms_norm(x, v, residual=dual(x)), "rms_norm_i8": lambda: qnn.rms_norm_i8(dual(x), v),
        "backward dy": lambda: qnn.rms_norm_backward(dual(x), x, v, rstd), "backward h": lambda: qnn.rms_norm_backward(x, dual(x), v, rstd),
        "backward rstd": lambda: qnn.rms_norm_backward(x, x, v, dual(rstd)), "backward dh": lambda: qnn.rms_norm_backward(x, x, v, rstd, dual(x)),
        "i8_quantize": lambda: qnn.i8_quantize(dual(x)), "i8_decode": lambda: qnn.i8_decode(qnn.I8Rows(codes, dual(scales))),
        "i8_gemm": lambda: qnn.i8_gemm(rows, qnn.I8Rows(codes, dual(scales))), "i8_gemm bias": lambda: qnn.i8_gemm(rows, rows, bias=dual(t.randn(4))),
        "route": lambda: qnn.route(dual(x), 2), "route bias": lambda: qnn.route(x, 2, bias=dual(v)),
        "route_backward": lambda: qnn.route_backward(t.zeros(4, 2), dual(x), ints), "route_backward dweights": lambda: qnn.route_backward(dual(t.zeros(4, 2)), x, ints),
        "g4_matvec": lambda: qnn.g4_matvec(dual(x), weights), "g4_expert_gemm": lambda: qnn.g4_expert_gemm(dual(x), weights, offsets),
        "expert_gemm_backward_weights": lambda: qnn.expert_gemm_backward_weights(dual(x), x, offsets),
    }


def test_tangents_are_refused(t, qnn):
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        for name, call in calls(t, qnn, lambda v: forward_ad.make_dual(v, t.ones_like(v))).items():
            with pytest.raises(ValueError, match="tangent"):
                call()
            with forward_ad._set_fwd_grad_enabled(False), pytest.raises(ValueError) as refusal:      # nothing is dropped then
                call()
            assert "tangent" not in str(refusal.value), name
    for name, call in calls(t, qnn, lambda v: v).items():
        with pytest.raises(ValueError) as refusal:                  # (these operands are on the host)
            call()
        assert "tangent" not in str(refusal.value), name

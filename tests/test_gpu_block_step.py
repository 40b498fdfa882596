"""A training step of the feed-forward block: what it does to every parameter and to the packed weights, and batches of one token and of
padding alone."""
import pytest

from test_gpu_block import DEV, HIDDEN, TOKENS, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_step_moves_every_parameter_by_its_gradient(t, qnn, dtype):
    block, x, residual = make(t, dtype)
    target = t.randn((TOKENS, HIDDEN), device=DEV, generator=t.Generator(device=DEV).manual_seed(5))
    names = ("w1", "w2", "up", "down", "router", "gain")
    packed = ("q1", "q2", "q_up", "q_down")
    rate = 3.0
    for _ in range(2):
        before = {n: getattr(block, n).clone() for n in names}
        codes = {n: getattr(block, n).codes.clone() for n in packed}
        out, saved = block.forward(x, residual)
        diff = out.float() - target
        grads = block.backward(diff / TOKENS, saved)
        loss = block.train_step(x, residual, target, rate)
        assert loss == float(0.5 * diff.square().sum(1).mean())
        for n in names:                                               # (every call repeats its bits, so the step's gradients are these)
            want = (before[n].float() - rate * grads[n]).to(before[n].dtype)
            assert t.equal(getattr(block, n), want) and not t.equal(want, before[n]), n
        fresh = {"q1": qnn.g4_pack_weights(block.w1, block.group), "q2": qnn.g4_pack_weights(block.w2, block.group),
                 "q_up": qnn.i8_quantize(block.up), "q_down": qnn.i8_quantize(block.down)}
        for n in packed:
            got = getattr(block, n)
            assert all(t.equal(a, b) for a, b in zip(got, fresh[n]) if isinstance(a, t.Tensor)) and not t.equal(got.codes, codes[n]), n
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_one_token_and_padding_alone(t, qnn, dtype):
    block, x, residual = make(t, dtype)
    out, saved = block.forward(x[:1], residual[:1])
    grads = block.backward(out, saved)
    assert all(bool(g.isfinite().all()) for g in grads.values()) and int((grads["w1"].flatten(1).abs().amax(1) > 0).sum()) == block.top
    out, saved = block.forward(x, residual, t.zeros(TOKENS, dtype=t.bool, device=DEV))
    routes = saved[7]
    assert int(routes.offsets[-1]) == 0 and bool((routes.place == -1).all())
    grads = block.backward(out, saved)
    assert all(bool((grads[n] == 0).all()) for n in ("w1", "w2", "router"))
    assert all(bool(g.isfinite().all()) and bool((g != 0).any()) for n, g in grads.items() if n not in ("w1", "w2", "router"))

"""Routing, norm, products in 8 bits and the 4-bit experts together, as run_case's feed-forward block uses them: against the same block
in 64 bits on the decoded weights, with torch's autograd for the gradients (straight through every rounding)."""
import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOKENS, HIDDEN, INNER, EXPERTS, TOP, GROUPS = 150, 200, 104, 24, 4, 4


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def make(t, dtype, seed=3):
    from paper_2106_09886_b200.run_case import FeedForwardBlock
    block = FeedForwardBlock(HIDDEN, INNER, EXPERTS, TOP, GROUPS, dtype=ref.torch_type(dtype), seed=seed)
    g = t.Generator(device=DEV).manual_seed(seed + 1)
    x, residual = (t.randn((TOKENS, HIDDEN), device=DEV, generator=g).to(ref.torch_type(dtype)) for _ in range(2))
    return block, x, residual


def decoded(t, qnn, w):
    """4-bit weights in 64 bits: the identity's rows through the product, exactly (one code times its scales in each sum)."""
    eye = t.eye(w.k, device=DEV)
    out = []
    for e in range(w.codes.shape[0]):
        one = w._replace(codes=w.codes[e:e + 1], scales=w.scales[e:e + 1], alpha=w.alpha[e:e + 1])
        out.append(qnn.g4_matvec(eye, one).t())
    return t.stack(out).double()


def plain(t, qnn, block, x, residual, mask, saved):
    """The block in 64 bits with leaves that take gradients.  The 8-bit activations enter with the values that the codes stand for
    (their roundings are the operator's own, tested by themselves) and pass gradients straight through; the choice of experts is the
    call's, checked against 64 bits by itself."""
    rows, y8, h8, rstd, a8, act8, logits, routes, *_ = saved
    leaf = lambda v: v.double().requires_grad_()
    p = {"x": leaf(x), "gain": leaf(block.gain), "router": leaf(block.router), "up": leaf(qnn.i8_decode(block.q_up, t.float32)),
         "down": leaf(qnn.i8_decode(block.q_down, t.float32)), "w1": decoded(t, qnn, block.q1).requires_grad_(),
         "w2": decoded(t, qnn, block.q2).requires_grad_()}
    through = lambda value, codes: value + (qnn.i8_decode(codes, t.float32).double() - value).detach()
    silu = t.nn.functional.silu
    h = p["x"] + residual.double()
    y = h / t.sqrt(h.square().mean(1, keepdim=True) + block.eps) * p["gain"]
    act = through(silu(through(y, rows) @ p["up"].t()), act8)
    out = h + act @ p["down"].t()
    score = t.sigmoid(y @ p["router"].t())
    chosen = routes.experts.long()
    s = t.where(chosen >= 0, score.gather(1, chosen.clamp(min=0)), 0.0)
    total = s.sum(1, keepdim=True)
    weight = block.factor * s / t.where(total > 0, total, 1.0)
    for i in range(TOP):
        e = chosen[:, i].clamp(min=0)
        z = t.einsum("thi,ti->th", p["w2"][e], silu(t.einsum("tih,th->ti", p["w1"][e], y)))
        out = out + z * weight[:, i:i + 1]
    return out, p


# fp32: sums of at most 208 products and a few products in a row, each to 2^-24 or, by the experts' weights, in three parts; errors of
# that size pass through some ten such layers: 1e-5 of the 2-norm.  16-bit types round every intermediate row to 2^-9 (2^-12), some
# ten in a row, the gradients as often again: 20 * 2^-9 (2^-12).
BOUND = {"fp32": 1e-5, "bf16": 20 * 2.0 ** -9, "fp16": 20 * 2.0 ** -12}


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("padded", [False, True])
def test_block_and_its_gradients(t, qnn, dtype, padded):
    block, x, residual = make(t, dtype)
    mask = None
    if padded:
        mask = t.ones(TOKENS, dtype=t.bool, device=DEV)
        mask[::7] = False
    out, saved = block.forward(x, residual, mask)
    routes = saved[7]
    want = ref.route(saved[6].cpu().double().numpy(), TOP, "sigmoid", block.bias.cpu().double().numpy(), GROUPS, GROUPS // 2, "top2", True, block.factor,
                     None if mask is None else mask.cpu().numpy())
    assert np.array_equal(routes.experts.cpu().numpy(), want[0]) and np.array_equal(routes.order.cpu().numpy(), want[2])
    exact, p = plain(t, qnn, block, x, residual, mask, saved)
    assert bool(out.isfinite().all())
    assert float((out.double() - exact.detach()).norm() / exact.detach().norm()) <= BOUND[dtype]
    g = t.Generator(device=DEV).manual_seed(9)
    dout = t.randn((TOKENS, HIDDEN), device=DEV, generator=g).to(x.dtype)
    (exact * dout.double()).sum().backward()
    grads = block.backward(dout, saved)
    for name, leaf in p.items():
        got = grads[name].double()
        assert got.shape == leaf.grad.shape and float((got - leaf.grad).norm() / leaf.grad.norm()) <= BOUND[dtype], name
    assert qnn.tensor_path_status() == 0


def test_block_repeats_its_bits_and_replays(t, qnn):
    """The same bits every time, captured or not, with inputs that change between replays; one token at a time as well."""
    block, x, residual = make(t, "bf16")
    first = block.forward(x, residual)[0]
    for _ in range(5):
        assert t.equal(block.forward(x, residual)[0], first)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        out = block.forward(x, residual)[0]
        one = block.forward(x[:1], residual[:1])[0]
    for _ in range(3):
        x.normal_()
        graph.replay()
        assert t.equal(out, block.forward(x, residual)[0]) and t.equal(one, block.forward(x[:1], residual[:1])[0])
    assert qnn.tensor_path_status() == 0


def test_block_trains(t, qnn):
    block, x, residual = make(t, "bf16")
    target = t.randn((TOKENS, HIDDEN), device=DEV)
    losses = [block.train_step(x, residual, target, 0.05) for _ in range(3)]
    assert all(np.isfinite(losses)) and qnn.tensor_path_status() == 0


def test_block_command(capsys, monkeypatch):
    import json
    from paper_2106_09886_b200 import run_case
    monkeypatch.setattr("sys.argv", ["run_case", "block", "--tokens", "40", "--experts", "8", "--top", "2", "--groups", "2", "--hidden", "128",
                                     "--inner", "64", "--reps", "2", "--warmup", "1"])
    run_case.main()
    r = json.loads(capsys.readouterr().out)
    assert r["call"] == "block" and r["status"] == 0 and r["forward_ms"] > 0

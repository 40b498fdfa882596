"""Routing on the GPU: the choice and the plan equal to 64 bits', weights and gradients within the bounds of layer_reference."""
import numpy as np
import pytest

import layer_reference as ref

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


def check(t, qnn, logits, top, mask=None, bias=None, **kw):
    """logits: a tensor on the GPU; bias and mask: numpy."""
    got = qnn.route(logits, top, mask=None if mask is None else t.from_numpy(mask).to(DEV), bias=None if bias is None else t.from_numpy(bias).to(DEV), **kw)
    l64 = logits.cpu().double().numpy()
    experts, weights, order, place, offsets = ref.route(l64, top, mask=mask, bias=None if bias is None else bias.astype(np.float64), **kw)
    assert np.array_equal(got.experts.cpu().numpy(), experts)
    assert np.array_equal(got.offsets.cpu().numpy(), offsets)
    assert np.array_equal(got.order.cpu().numpy(), order) and np.array_equal(got.place.cpu().numpy(), place)
    w = got.weights.cpu().double().numpy()
    nan = np.isnan(weights)
    assert np.array_equal(np.isnan(w), nan)
    bound = ref.weight_bound(weights, l64, top, kw.get("score", "softmax"), kw.get("renormalise", True))
    assert np.all(np.abs(w - weights)[~nan] <= bound[~nan])
    return got


def logits_of(t, rng, tokens, experts, dtype="fp32", size=1.5):
    v = rng.standard_normal((tokens, experts)) * size + 0.5 * rng.standard_normal(experts)
    return t.from_numpy(v.astype(np.float32)).to(ref.torch_type(dtype)).to(DEV)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("tokens,experts,top", [(1, 1, 1), (1, 64, 6), (3, 8, 2), (64, 33, 5), (65, 32, 32), (200, 256, 8), (513, 8, 2), (700, 160, 6), (130, 512, 10),
                                                (70, 1024, 4), (5, 1000, 32), (2000, 5, 1)])
def test_route(t, qnn, score, biased, tokens, experts, top):
    rng = np.random.default_rng(tokens * 10007 + experts * 31 + top + biased)
    bias = (rng.standard_normal(experts) * 0.05).astype(np.float32) if biased else None
    logits = logits_of(t, rng, tokens, experts)
    mask = rng.random(tokens) < 0.8
    check(t, qnn, logits, top, bias=bias, score=score)
    check(t, qnn, logits, top, bias=bias, score=score, renormalise=False, factor=2.5, mask=mask)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("biased", [False, True])
def test_route_narrow_types(t, qnn, dtype, biased):
    """Logits of few bits: many are equal, and the lowest expert goes first."""
    rng = np.random.default_rng(7)
    bias = (rng.integers(0, 3, 128) * 0.25).astype(np.float32) if biased else None
    for score in ("softmax", "sigmoid"):
        check(t, qnn, logits_of(t, rng, 150, 128, dtype), 8, bias=bias, score=score)
        check(t, qnn, logits_of(t, rng, 150, 128, dtype).round(), 8, bias=bias, score=score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("experts,groups,top_groups,top", [(256, 8, 4, 8), (60, 4, 1, 6), (64, 32, 7, 9), (24, 3, 2, 16), (40, 20, 20, 5), (1024, 2, 1, 8), (1024, 32, 3, 12), (6, 2, 1, 3)])
def test_groups(t, qnn, score, biased, group_score, experts, groups, top_groups, top):
    rng = np.random.default_rng(experts + groups + top)
    bias = (rng.standard_normal(experts) * 0.1).astype(np.float32) if biased else None
    for tokens in (3, 150):
        check(t, qnn, logits_of(t, rng, tokens, experts), top, bias=bias, score=score, groups=groups, top_groups=top_groups, group_score=group_score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_keys_nearer_than_fp32_can_tell(t, qnn, score, groups):
    """Biases that make every key of a token the same number within fp32's rounding: the choice is that of 64 bits."""
    rng = np.random.default_rng(11)
    experts, top = 64, 8
    row = rng.standard_normal((1, experts)).astype(np.float32)
    s = ref.scores(row.astype(np.float64), score)[0]
    bias = (0.75 - s).astype(np.float32)
    keys = s + bias.astype(np.float64)
    assert np.max(np.abs(keys - 0.75)) < 2.0 ** -24 and np.min(np.abs(np.diff(np.sort(keys)))) > 1e-12      # (64 bits tell them apart)
    logits = t.from_numpy(np.repeat(row, 100, 0)).to(DEV)
    for group_score in ("max", "top2"):
        check(t, qnn, logits, top, bias=bias, score=score, groups=groups, top_groups=max(1, groups // 2), group_score=group_score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top", [(64, 8), (256, 8), (256, 31), (256, 32), (40, 1), (20, 12), (1000, 6)])
def test_keys_near_one_another_in_places(t, qnn, score, experts, top):
    """Keys that fp32 cannot tell apart in pairs, in fours, and in one run of twenty, among keys that it can; with and without a bias."""
    rng = np.random.default_rng(experts + top)
    for size in (2, 4, 20):
        if size > experts:
            continue
        rows, biases = [], []
        row = rng.standard_normal(experts).astype(np.float32)
        s = ref.scores(row[None].astype(np.float64), score)[0]
        place = rng.permutation(experts)
        target = 0.2 + 0.6 * np.arange((experts + size - 1) // size)[np.argsort(np.argsort(place)) // size] / experts
        bias = (target - s).astype(np.float32)
        check(t, qnn, t.from_numpy(np.repeat(row[None], 40, 0)).to(DEV), top, bias=bias, score=score)
        check(t, qnn, t.from_numpy(np.repeat(row[None], 40, 0)).to(DEV), top, bias=bias, score=score, groups=4, top_groups=4, group_score="top2")
        # without a bias: logits that differ in their lowest bits only
        base = np.repeat(rng.standard_normal((40, (experts + size - 1) // size)), size, 1)[:, :experts].astype(np.float32)
        bits = base.view(np.int32) + rng.integers(0, 6, base.shape).astype(np.int32)
        l = np.take_along_axis(bits.view(np.float32), rng.permuted(np.tile(np.arange(experts), (40, 1)), axis=1), 1)
        check(t, qnn, t.from_numpy(np.ascontiguousarray(l)).to(DEV), top, score=score)


def test_excluded_experts_and_tokens(t, qnn):
    """Masked experts, rows that a mask leaves nothing of, NaN and infinities."""
    rng = np.random.default_rng(13)
    inf = float("inf")
    for score in ("softmax", "sigmoid"):
        for bias in (None, (rng.standard_normal(40) * 0.1).astype(np.float32)):
            for groups in (1, 4):
                l = logits_of(t, rng, 100, 40)
                l[:, 5:9] = -inf                                      # experts that nobody gets
                l[3] = -inf                                           # a row of nothing
                l[4] = -inf
                l[4, 17] = -3.0                                       # one expert left, fewer than top
                l[5, 39] = float("nan")
                l[6, 0] = inf
                l[7] = t.finfo(t.float32).min                         # a mask's lowest value in every place
                l[8, :39] = t.finfo(t.float32).min
                l[9] = -200.0                                         # scores that underflow
                l[9, 12] = -190.0
                b = bias
                if bias is not None:
                    b = bias.copy()
                    b[20], b[21] = -inf, np.nan
                mask = np.ones(100, dtype=bool)
                mask[50:60] = False
                check(t, qnn, l, 6, mask=mask, bias=b, score=score, groups=groups, top_groups=max(1, groups // 2))
                got = check(t, qnn, l, 6, mask=mask, bias=b, score=score, groups=groups, top_groups=max(1, groups // 2), group_score="top2")
                assert got.experts[3].tolist() == [-1] * 6 and got.weights[3].tolist() == [0.0] * 6 and got.experts[50].tolist() == [-1] * 6
    none = np.zeros(100, dtype=bool)
    got = check(t, qnn, l, 6, mask=none)
    assert int(got.offsets[-1]) == 0 and bool((got.order == -1).all())


def test_signed_zeros_are_equal(t, qnn):
    l = t.zeros((4, 16), device=DEV)
    l[:, ::2] = -0.0
    assert qnn.route(l, 4).experts.tolist() == [[0, 1, 2, 3]] * 4


def test_strides_types_of_mask_and_no_tokens(t, qnn):
    rng = np.random.default_rng(17)
    big = logits_of(t, rng, 90, 100, "bf16")
    a, b = qnn.route(big[:, 3:67], 4), qnn.route(big[:, 3:67].contiguous(), 4)
    assert all(t.equal(x, y) for x, y in zip(a, b))
    mask = t.from_numpy(rng.random(90) < 0.5).to(DEV)
    assert all(t.equal(x, y) for x, y in zip(qnn.route(big, 4, mask=mask), qnn.route(big, 4, mask=mask.to(t.uint8) * 3)))
    none = qnn.route(big[:0], 4)
    assert none.experts.shape == (0, 4) and none.offsets.tolist() == [0] * 101


def test_many_tokens(t, qnn):
    """The plan over many runs, against a stable sort."""
    g = t.Generator(device=DEV).manual_seed(5)
    l = t.randn((40001, 96), device=DEV, generator=g)
    l[:, 7] += 3
    r = qnn.route(l, 5)
    flat = r.experts.reshape(-1).long()
    assert t.equal(r.order.long(), flat.sort(stable=True).indices)
    counts = t.bincount(flat, minlength=96)
    assert t.equal(r.offsets[1:].long(), counts.cumsum(0)) and r.offsets[0].item() == 0
    assert t.equal(r.order[r.place.reshape(-1).long()], t.arange(flat.numel(), device=DEV, dtype=t.int32))
    want = l.topk(5, 1)
    assert t.equal(want.indices.int(), r.experts)


@pytest.mark.parametrize("experts,top", [(5, 2), (64, 6), (100, 8), (200, 4), (600, 3)])
def test_every_split_of_few_tokens(t, qnn, experts, top):
    """One block, clusters of two to eight whose last blocks have fewer tokens or none, and the two and three launches beyond: against a
    stable sort."""
    g = t.Generator(device=DEV).manual_seed(experts)
    for tokens in (1, 2, 7, 8, 9, 15, 16, 17, 18, 25, 31, 33, 34, 41, 49, 57, 63, 64, 65, 66, 73, 97, 100, 121, 127, 128, 129, 200, 255, 256, 257, 300, 1000):
        l = t.randn((tokens, experts), device=DEV, generator=g)
        mask = t.rand(tokens, device=DEV, generator=g) < 0.9
        r = qnn.route(l, top, mask=mask)
        assert t.equal(r.experts, t.where(mask.view(-1, 1), l.topk(top, 1).indices.int(), -1))
        flat = r.experts.reshape(-1).long()
        key = t.where(flat < 0, experts, flat)
        rows = int((flat >= 0).sum())
        assert t.equal(r.offsets.long(), t.cat([t.zeros(1, dtype=t.int64, device=DEV), t.bincount(key, minlength=experts + 1)[:experts].cumsum(0)]))
        assert t.equal(r.order[:rows].long(), key.sort(stable=True).indices[:rows]) and bool((r.order[rows:] == -1).all())
        place = t.full((tokens * top,), -1, dtype=t.int32, device=DEV)
        place[r.order[:rows].long()] = t.arange(rows, dtype=t.int32, device=DEV)
        assert t.equal(r.place.reshape(-1), place)


# ------------------------------------------------------------------------------------------------ backward

@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("tokens,experts,top", [(1, 1, 1), (3, 8, 2), (40, 33, 5), (20, 32, 32), (50, 256, 8), (9, 1000, 32), (300, 160, 6)])
def test_backward(t, qnn, dtype, score, renormalise, tokens, experts, top):
    rng = np.random.default_rng(tokens + experts + top)
    logits = logits_of(t, rng, tokens, experts, dtype)
    l64 = logits.cpu().double().numpy()
    chosen = ref.route(l64, top, score=score, mask=rng.random(tokens) < 0.9)[0].astype(np.int32)
    chosen[0, top - 1] = -1
    dw = rng.standard_normal((tokens, top)).astype(np.float32)
    got = qnn.route_backward(t.from_numpy(dw).to(DEV), logits, t.from_numpy(chosen).to(DEV), score, renormalise, 1.5)
    want, size = ref.route_backward(dw.astype(np.float64), l64, chosen, score, renormalise, 1.5)
    err = np.abs(got.cpu().double().numpy() - want)
    assert got.dtype == logits.dtype and np.all(err <= ref.route_backward_bound(want, size, l64, dtype))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_backward_against_differences(t, qnn, score, renormalise):
    rng = np.random.default_rng(3)
    l = rng.standard_normal((2, 12)).astype(np.float32)
    dw = rng.standard_normal((2, 4)).astype(np.float32)
    chosen = np.array([[3, 0, 7, 11], [1, 2, 9, -1]], dtype=np.int32)
    got = qnn.route_backward(t.from_numpy(dw).to(DEV), t.from_numpy(l).to(DEV), t.from_numpy(chosen).to(DEV), score, renormalise, 2.0).cpu().double().numpy()

    def f(l):
        s, total = ref.scores(l, score), 0.0
        for r in range(2):
            pick = [e for e in chosen[r] if e >= 0]
            w = 2.0 * s[r][pick] / (s[r][pick].sum() if renormalise else 1.0)
            total += (w * dw[r][:len(pick)]).sum()
        return total
    for r in range(2):
        for e in range(12):
            step = np.zeros((2, 12))
            step[r, e] = 1e-5
            l64 = l.astype(np.float64)
            assert abs((f(l64 + step) - f(l64 - step)) / 2e-5 - got[r, e]) < 1e-6 * 5


def test_backward_strange_choices(t, qnn):
    """The same expert twice counts twice; experts that do not exist count as none; rows around the result stay."""
    rng = np.random.default_rng(5)
    logits = logits_of(t, rng, 4, 20)
    chosen = np.array([[1, 1, 5], [20, 3, -7], [-1, -1, -1], [2 ** 31 - 1, 0, 19]], dtype=np.int32)
    dw = rng.standard_normal((4, 3)).astype(np.float32)
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            out = t.full((6, 24), 4.0, device=DEV)
            qnn.route_backward(t.from_numpy(dw).to(DEV), logits, t.from_numpy(chosen).to(DEV), score, renormalise, out=out[1:5, 2:22])
            want, size = ref.route_backward(dw.astype(np.float64), logits.cpu().double().numpy(), chosen, score, renormalise)
            got = out[1:5, 2:22].cpu().double().numpy()
            assert np.all(np.abs(got - want) <= ref.route_backward_bound(want, size, logits.cpu().double().numpy(), "fp32"))
            out[1:5, 2:22] = 4.0
            assert bool((out == 4.0).all())


def test_captured(t, qnn):
    g = t.Generator(device=DEV).manual_seed(9)
    for tokens in (20, 500):
        l, bias = t.randn((tokens, 64), device=DEV, generator=g), t.randn(64, device=DEV, generator=g) * 0.1
        dw = t.randn((tokens, 6), device=DEV, generator=g)
        def step():
            r = qnn.route(l, 6, "sigmoid", bias, 8, 4, "top2")
            return tuple(r) + (qnn.route_backward(dw, l, r.experts, "sigmoid"),)
        step()
        t.cuda.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            out = step()
        for _ in range(3):
            l.normal_()
            graph.replay()
            for a, b in zip(out, step()):
                assert t.equal(a, b)


def test_refusals(t, qnn):
    l = t.randn((4, 40), device=DEV)
    for bad in (lambda: qnn.route(l, 2, score="tanh"), lambda: qnn.route(l, 2, group_score="mean"), lambda: qnn.route(l, 2, bias=t.zeros(39, device=DEV)),
                lambda: qnn.route(l, 2, bias=t.zeros(40)), lambda: qnn.route(l, 2, mask=t.ones(3, dtype=t.bool, device=DEV)),
                lambda: qnn.route(l, 2, mask=t.ones(4, device=DEV)), lambda: qnn.route(l.double(), 2), lambda: qnn.route(l.cpu(), 2),
                lambda: qnn.route(l.clone().requires_grad_(), 2), lambda: qnn.route(l.t(), 2),
                lambda: qnn.route_backward(t.zeros((4, 2), device=DEV), l, t.zeros((4, 2), device=DEV)),
                lambda: qnn.route_backward(t.zeros((4, 2), device=DEV), l, t.zeros((4, 3), dtype=t.int32, device=DEV)),
                lambda: qnn.route_backward(t.zeros((3, 2), device=DEV), l, t.zeros((3, 2), dtype=t.int32, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qnn.route(l, 0), lambda: qnn.route(l, 33), lambda: qnn.route(l, 41), lambda: qnn.route(l, 2, groups=3), lambda: qnn.route(l, 2, groups=0),
                lambda: qnn.route(l, 2, groups=4, top_groups=5), lambda: qnn.route(l, 11, groups=4, top_groups=1),
                lambda: qnn.route(l, 2, groups=40, top_groups=2), lambda: qnn.route(l, 2, factor=float("nan")),
                lambda: qnn.route(t.zeros((1, 1025), device=DEV), 2)):
        with pytest.raises(qnn.QnnError):
            bad()

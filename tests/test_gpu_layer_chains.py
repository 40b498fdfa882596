"""Norm, products in 8 bits, routing and their gradients one behind another with nothing between them, each reading what the one before
has just written (their kernels start while the ones ahead still run); on two streams at once; and around their results."""
import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUNDS = 10


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def chain(t, qnn, dtype, width, experts, seed):
    """A step through every call, and the inputs of ROUNDS steps; `wait` runs between calls."""
    g = t.Generator(device=DEV).manual_seed(seed)
    kind = ref.torch_type(dtype)
    real = lambda *shape: t.randn(shape, device=DEV, generator=g).to(kind)
    gain, up, head = 1 + 0.1 * real(width), qnn.i8_quantize(real(width, width)), qnn.i8_quantize(real(experts, width))
    bias = t.randn(experts, device=DEV, generator=g) * 0.05

    def step(x, residual, wait):
        rows, y, h, rstd = qnn.rms_norm_i8(x, gain, 1e-6, residual, both=True)
        wait()
        a = qnn.i8_gemm(rows, up, kind)
        wait()
        again = qnn.i8_quantize(a)
        wait()
        logits = qnn.i8_gemm(again, head, t.float32)
        wait()
        routes = qnn.route(logits, 4, "sigmoid", bias, 2, 1, "top2")
        wait()
        dlogits = qnn.route_backward(routes.weights, logits, routes.experts, "sigmoid")
        wait()
        back = qnn.i8_decode(again, kind)
        wait()
        dx, dgain = qnn.rms_norm_backward(back, h, gain, rstd, a)
        wait()
        return [rows.codes, rows.scales, y, h, rstd, a, again.codes, logits, *routes, dlogits, back, dx, dgain]
    return step, real


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", [(1, 264), (1, 333), (20, 512), (90, 1001), (300, 264), (700, 1024)])
def test_chain(t, qnn, dtype, rows, width):
    step, real = chain(t, qnn, dtype, width, 40, rows + width)
    inputs = [(real(rows, width), real(rows, width)) for _ in range(ROUNDS)]
    want = [step(x, r, t.cuda.synchronize) for x, r in inputs]
    t.cuda.synchronize()
    for _ in range(2):
        got = [step(x, r, lambda: None) for x, r in inputs]
        t.cuda.synchronize()
        for a, b in zip(got, want):
            for u, v in zip(a, b):
                assert t.equal(u, v)
    assert qnn.tensor_path_status() == 0


def test_two_streams_at_once(t, qnn):
    steps = [chain(t, qnn, "bf16", 512, 64, seed) for seed in (1, 2)]
    inputs = [[(real(200, 512), real(200, 512)) for _ in range(ROUNDS)] for _, real in steps]
    want = [[step(x, r, t.cuda.synchronize) for x, r in some] for (step, _), some in zip(steps, inputs)]
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    t.cuda.synchronize()
    got = [[], []]
    for i in range(ROUNDS):
        for k in range(2):
            with t.cuda.stream(streams[k]):
                got[k].append(steps[k][0](*inputs[k][i], lambda: None))
    t.cuda.synchronize()
    for k in range(2):
        for a, b in zip(got[k], want[k]):
            assert all(t.equal(u, v) for u, v in zip(a, b))


def test_results_lie_apart(t, qnn):
    """Small results of one call share an allocation: each starts on 16 bytes and none overlaps another."""
    x, gain = t.randn((3, 100), device=DEV), t.ones(100, device=DEV)
    rows, y, h, rstd = qnn.rms_norm_i8(x, gain, 1e-6, x, both=True)
    routes = qnn.route(t.randn((3, 30), device=DEV), 3)
    for results in ([rows.codes, rows.scales, y, h, rstd], list(routes), list(qnn.i8_quantize(x)), list(qnn.rms_norm_backward(y, h, gain, rstd))):
        spans = sorted((r.data_ptr(), r.data_ptr() + ((r.shape[0] - 1) * r.stride(0) + (r.shape[1] if r.dim() > 1 else 1)) * r.element_size()) for r in results)
        assert all(a % 16 == 0 for a, _ in spans) and all(b <= c for (_, b), (c, _) in zip(spans, spans[1:]))


def test_c_calls_write_their_results_alone(t, qnn):
    """Bands around every result of the C calls stay as they were, and so do codes behind a row's width."""
    import ctypes as C
    p = lambda v: C.c_void_p(v.data_ptr())
    stream = C.c_void_p(t.cuda.current_stream().cuda_stream)
    for rows, width in ((3, 40), (2, 257), (5, 1000)):
        x, gain = t.randn((rows, width), device=DEV), t.ones(width, device=DEV)
        ldc = (width + 15) // 16 * 16 + 32
        codes, scales, y, rstd = (t.full(s, 5, dtype=d, device=DEV) for s, d in (((rows + 2, ldc), t.int8), ((rows + 2,), t.float32), ((rows + 2, width + 3), t.float32), ((rows + 2,), t.float32)))
        at = lambda v, n: C.c_void_p(v.data_ptr() + n * v.element_size())
        assert qnn.lib.qnn_rms_norm(p(x), 0, rows, width, width, None, 0, p(gain), 0, 1e-6, None, 0, at(y, width + 3), width + 3, at(codes, ldc), ldc, at(scales, 1), at(rstd, 1), stream) == 0
        q, h, r = qnn.rms_norm_i8(x, gain)
        # (rows of y that lie off 16 bytes are normed element by element, in another order of the sum than the call beside it: each is off
        # by the reference's count of roundings at most, and a code by one where a quotient lies next to a half)
        near = lambda a, b, n: bool(((a - b).abs() <= 2 * n * ref.U32 * b.abs()).all())
        assert near(scales[1:rows + 1], q.scales, ref.Y_ROUNDINGS + 1) and near(rstd[1:rows + 1], r, ref.RSTD_ROUNDINGS)
        assert int((codes[1:rows + 1, :width].int() - q.codes.int()).abs().max()) <= 1
        codes[1:rows + 1, :width] = 5
        y[1:rows + 1, :width] = 5
        scales[1:rows + 1] = 5
        rstd[1:rows + 1] = 5
        assert all(bool((v == 5).all()) for v in (codes, y, scales, rstd))
    for tokens in (3, 100, 5000):
        l = t.randn((tokens, 24), device=DEV)
        n = tokens * 3
        chosen, weights, order, place, offsets = (t.full((s,), 5, dtype=d, device=DEV) for s, d in ((n + 8, t.int32), (n + 8, t.float32), (n + 8, t.int32), (n + 8, t.int32), (33, t.int32)))
        need = qnn.lib.qnn_route_workspace(tokens, 24, 3)
        ws = t.full((need + 256,), 5, dtype=t.uint8, device=DEV)
        assert qnn.lib.qnn_route(p(l), 0, tokens, 24, 24, 3, 2, None, 1, 1, 1.0, None, at(chosen, 4), at(weights, 4), at(order, 4), at(place, 4), at(offsets, 4),
                                 p(ws), need, stream) == 0
        r = qnn.route(l, 3)
        for got, want, size in ((chosen, r.experts, n), (weights, r.weights, n), (order, r.order, n), (place, r.place, n), (offsets, r.offsets, 25)):
            assert t.equal(got[4:4 + size], want.reshape(-1))
            got[4:4 + size] = 5
            assert bool((got == 5).all())
        assert bool((ws[need:] == 5).all())
        # the choice alone, without a plan
        assert qnn.lib.qnn_route(p(l), 0, tokens, 24, 24, 3, 2, None, 1, 1, 1.0, None, p(chosen), p(weights), None, None, None, None, 0, stream) == 0
        assert t.equal(chosen[:n], r.experts.reshape(-1)) and t.equal(weights[:n], r.weights.reshape(-1))


def test_equal_logits(t, qnn):
    """What a router of zeros gives: every expert the same, the lowest first; with a bias of zeros as well."""
    for experts, top in ((8, 2), (64, 6), (256, 8), (256, 32), (1000, 4)):
        l = t.zeros((500, experts), device=DEV)
        for bias in (None, t.zeros(experts, device=DEV)):
            for score in ("softmax", "sigmoid"):
                r = qnn.route(l, top, score, bias)
                assert t.equal(r.experts, t.arange(top, device=DEV, dtype=t.int32).expand(500, top))
                assert bool((r.weights - 1.0 / top).abs().max() < 1e-6)
    r = qnn.route(t.zeros((30, 64), device=DEV), 4, groups=8, top_groups=2, group_score="top2")
    assert r.experts.tolist() == [[0, 1, 2, 3]] * 30

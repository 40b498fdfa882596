"""Host side of the group-scaled 4-bit weight calls: sizes, refusals before any launch, and the storage format itself."""
import ctypes

import numpy as np
import pytest

import g4_reference as ref


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import build
    build.build()
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 8192)()
    test_buffer = ctypes.c_void_p((ctypes.addressof(buf) + 255) // 256 * 256)      # aligned, never read by these calls
    test_buffer.keep = buf
    return test_buffer


def test_sizes(qnn):
    f, g = qnn.lib.qnn_g4_codes_bytes, qnn.lib.qnn_g4_scales_bytes
    for n, k in [(1, 1), (128, 128), (129, 128), (777, 1000), (4096, 4096)]:
        assert f(1, n, k) == ref.tiles(n) * ref.tiles(k) * 8192 and f(3, n, k) == 3 * f(1, n, k)
        for group in (32, 64, 128):
            assert g(2, n, k, group) == 2 * ref.tiles(n) * ref.tiles(k) * 128 * 128 // group
    assert f(1, 4096, 4096) * 2 == 4096 * 4096
    assert f(0, 4, 4) == 0 and f(1, 0, 4) == 0 and f(1, 4, -1) == 0 and f(4097, 4, 4) == 0 and f(1, 65535 * 16 + 1, 4) == 0
    assert g(1, 4, 4, 16) == 0 and g(1, 4, 4, 0) == 0 and g(1, 4, 0, 32) == 0


def test_format_round_trip():
    rng = np.random.default_rng(3)
    for n, k, group in [(1, 1, 32), (130, 129, 64), (5, 300, 128), (257, 96, 32)]:
        w = (rng.standard_normal((n, k)) * 0.02).astype(np.float32)
        t, byte, alpha = ref.quantize(w, group)
        codes, scales = ref.store(t, byte, group)
        got = ref.decode(codes, scales, alpha, n, k, group)
        step = np.repeat(float(alpha) * ref.e4m3_values()[byte], group, axis=1)[:, :k]
        # a scale is off by at most 1/16 of itself, so the largest weight of a group stays within one unit of code 15
        assert np.all(np.abs(got - w) <= 1.0001 * step + 2.0 ** -9 * 15 * float(alpha))


def test_pack_refusals(qnn, p):
    f = qnn.lib.qnn_g4_pack_weights
    mis = ctypes.c_void_p(p.value + 4)
    ok = (p, 0, 1, 4, 64, 64, 32, p, p, p, None)

    def call(**kw):
        names = ("w", "type", "experts", "n", "k", "ldw", "group", "codes", "scales", "alpha", "stream")
        return f(*[kw.get(name, v) for name, v in zip(names, ok)])

    for bad in ({"w": None}, {"codes": None}, {"scales": None}, {"alpha": None}, {"type": 3}, {"type": -1}, {"experts": 0},
                {"n": 0}, {"k": 0}, {"ldw": 63}, {"group": 16}, {"group": 0}, {"group": 256}, {"n": 65535 * 16 + 1}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"codes": mis}, {"scales": mis}, {"w": ctypes.c_void_p(p.value + 2)}, {"alpha": ctypes.c_void_p(p.value + 1)},
                {"type": 1, "w": ctypes.c_void_p(p.value + 1)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(experts=4096, n=65535 * 16, k=65535 * 16, ldw=65535 * 16) == qnn.E_RANGE


def test_matvec_refusals(qnn, p):
    f = qnn.lib.qnn_g4_matvec
    mis = ctypes.c_void_p(p.value + 4)
    ok = (p, 1, 2, 64, p, p, p, 8, 64, 32, p, 8, None, 0, None)

    def call(**kw):
        names = ("x", "type", "rows", "ldx", "codes", "scales", "alpha", "n", "k", "group", "y", "ldy", "ws", "ws_bytes", "stream")
        return f(*[kw.get(name, v) for name, v in zip(names, ok)])

    for bad in ({"x": None}, {"y": None}, {"codes": None}, {"scales": None}, {"alpha": None}, {"type": 7}, {"rows": -1},
                {"ldx": 63}, {"ldy": 7}, {"group": 48}, {"n": 0}, {"k": -5}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"codes": mis}, {"scales": mis}, {"x": ctypes.c_void_p(p.value + 1)}, {"type": 0, "y": ctypes.c_void_p(p.value + 2)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(rows=1 << 31) == qnn.E_RANGE
    assert call(rows=0) == qnn.OK and call(rows=0, x=None, y=None) == qnn.OK       # nothing to do, nothing launched
    assert call(rows=0, group=48) == qnn.E_ARG
    need = qnn.lib.qnn_g4_matvec_workspace(p, 0, 200, 64, 8, 64)
    assert need > 0 and call(type=0, rows=200) == qnn.E_ARG and call(type=0, rows=200, ws=p, ws_bytes=need - 1) == qnn.E_ARG
    assert call(type=0, rows=200, ws=mis, ws_bytes=need) == qnn.E_ALIGN


@pytest.mark.parametrize("name", ["qnn_g4_expert_gemm", "qnn_g4_expert_backward_data"])
def test_expert_refusals(qnn, p, name):
    f = getattr(qnn.lib, name)
    mis = ctypes.c_void_p(p.value + 4)
    forward = name == "qnn_g4_expert_gemm"
    width, other = (64, 8) if forward else (8, 64)
    ok = (p, 1, 2, width, p, 3, p, p, p, 8, 64, 32, p, other, p, 8192, None)

    def call(**kw):
        names = ("x", "type", "rows", "ldx", "offsets", "experts", "codes", "scales", "alpha", "n", "k", "group", "y", "ldy",
                 "ws", "ws_bytes", "stream")
        return f(*[kw.get(key, v) for key, v in zip(names, ok)])

    for bad in ({"x": None}, {"y": None}, {"codes": None}, {"scales": None}, {"alpha": None}, {"offsets": None}, {"type": 3},
                {"rows": -1}, {"experts": 0}, {"experts": 4097}, {"ldx": width - 1}, {"ldy": other - 1}, {"group": 1},
                {"n": 0}, {"k": 0}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"codes": mis}, {"scales": mis}, {"offsets": ctypes.c_void_p(p.value + 2)}, {"x": ctypes.c_void_p(p.value + 1)},
                {"y": ctypes.c_void_p(p.value + 1)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(rows=1 << 31) == qnn.E_RANGE
    assert call(rows=0) == qnn.OK and call(rows=0, x=None, y=None) == qnn.OK
    need = getattr(qnn.lib, name + "_workspace")(p, 0, 2, width + 1, 3, 8, 64)
    if need:                                                   # a workspace that is missing, too small or misaligned
        assert call(type=0, ldx=width + 1, ws=None, ws_bytes=0) == qnn.E_ARG
        assert call(type=0, ldx=width + 1, ws_bytes=need - 1) == qnn.E_ARG
        assert call(type=0, ldx=width + 1, ws=mis) == qnn.E_ALIGN


def test_weight_gradient_refusals(qnn, p):
    f = qnn.lib.qnn_expert_backward_weights
    ok = (p, p, 1, 2, 8, 64, p, 3, 8, 64, p, p, 8192, None)

    def call(**kw):
        names = ("dy", "x", "type", "rows", "lddy", "ldx", "offsets", "experts", "n", "k", "gw", "ws", "ws_bytes", "stream")
        return f(*[kw.get(key, v) for key, v in zip(names, ok)])

    for bad in ({"dy": None}, {"x": None}, {"gw": None}, {"offsets": None}, {"type": 3}, {"rows": -1}, {"experts": 0}, {"n": 0},
                {"k": 0}, {"lddy": 7}, {"ldx": 63}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"gw": ctypes.c_void_p(p.value + 2)}, {"offsets": ctypes.c_void_p(p.value + 2)}, {"x": ctypes.c_void_p(p.value + 1)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(rows=1 << 31) == qnn.E_RANGE
    need = qnn.lib.qnn_expert_backward_weights_workspace(p, p, 0, 2, 8, 64, 3, 8, 64)
    if need:
        assert call(type=0, ws=None, ws_bytes=0) == qnn.E_ARG
        assert call(type=0, ws_bytes=need - 1) == qnn.E_ARG
        assert call(type=0, ws=ctypes.c_void_p(p.value + 16)) == qnn.E_ALIGN


def test_binding_refusals(qnn):
    """The binding checks shapes, types and devices before it passes a pointer on."""
    import torch
    cpu = torch.zeros((2, 64))
    w = qnn.G4Weights(torch.zeros((1, 1, 1, 4, 128, 4), dtype=torch.int32), torch.zeros((1, 1, 1, 4, 128), dtype=torch.uint8),
                      torch.ones(1), 8, 64, 32)
    offsets = torch.tensor([0, 2], dtype=torch.int32)
    for call in (lambda: qnn.g4_matvec(cpu, w), lambda: qnn.g4_expert_gemm(cpu, w, offsets),
                 lambda: qnn.g4_expert_gemm_backward_data(torch.zeros((2, 8)), w, offsets),
                 lambda: qnn.expert_gemm_backward_weights(torch.zeros((2, 8)), cpu, offsets),
                 lambda: qnn.g4_pack_weights(torch.zeros((8, 64)))):
        with pytest.raises(ValueError):
            call()
    # shapes and types are looked at before devices
    for bad, why in ((w._replace(group=16), "group"), (w._replace(n=129), "codes"), (w._replace(k=129), "codes"), (w._replace(n=0), "codes"),
                     (w._replace(codes=w.codes.float()), "codes"), (w._replace(scales=w.scales[..., :64].contiguous()), "scales"),
                     (w._replace(alpha=torch.ones(2)), "alpha"), (w._replace(codes=w.codes.expand(2, -1, -1, -1, -1, -1)), "codes"),
                     (w._replace(codes=None), "codes")):
        with pytest.raises(ValueError, match=why):
            qnn.g4_matvec(cpu, bad)
    for bad, why in ((torch.tensor([0, 2]), "offsets"), (torch.tensor([0], dtype=torch.int32), "offsets"),
                     (torch.zeros((2, 2), dtype=torch.int32), "offsets"), (torch.tensor([0, 1, 2], dtype=torch.int32), "experts"), (None, "offsets")):
        with pytest.raises(ValueError, match=why):
            qnn.g4_expert_gemm(cpu, w, bad)
    for bad in (cpu.double(), cpu[:, :63], cpu[0], cpu.expand(2, 2, 64), torch.zeros(64, 2).t(), cpu[:1].expand(4, 64), None):
        with pytest.raises(ValueError):
            qnn.g4_matvec(bad, w)
    with pytest.raises(ValueError, match="type"):
        qnn.expert_gemm_backward_weights(torch.zeros((2, 8)), cpu.bfloat16(), offsets)
    with pytest.raises(ValueError, match="current CUDA device"):
        qnn.g4_matvec(cpu, w)


def test_operands_that_require_grad_are_refused_while_gradients_are_recorded(qnn):
    """The calls record no gradients; a result without a graph must not come back as if nothing were missing."""
    import torch
    w = qnn.G4Weights(torch.zeros((1, 1, 1, 4, 128, 4), dtype=torch.int32), torch.zeros((1, 1, 1, 4, 128), dtype=torch.uint8),
                      torch.ones(1), 8, 64, 32)
    offsets = torch.tensor([0, 2], dtype=torch.int32)
    x, dy = torch.zeros((2, 64)), torch.zeros((2, 8))
    xg, dyg = torch.zeros((2, 64), requires_grad=True), torch.zeros((2, 8), requires_grad=True)
    calls = (lambda: qnn.g4_matvec(xg, w), lambda: qnn.g4_expert_gemm(xg, w, offsets), lambda: qnn.g4_expert_gemm(xg * 2, w, offsets),
             lambda: qnn.g4_expert_gemm_backward_data(dyg, w, offsets), lambda: qnn.expert_gemm_backward_weights(dyg, x, offsets),
             lambda: qnn.expert_gemm_backward_weights(dy, xg, offsets),
             lambda: qnn.g4_matvec(x, w._replace(alpha=torch.ones(1, requires_grad=True))))
    for call in calls:
        with pytest.raises(ValueError, match="record no gradients"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="device"):       # past that check, on to the next
            call()
    with pytest.raises(ValueError, match="device"):
        qnn.g4_matvec(xg.detach(), w)

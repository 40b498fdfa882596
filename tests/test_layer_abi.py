"""Host side of the routing, the norm and the rows in 8 bits: sizes and refusals before any launch, and the plain forms against
small cases done by hand."""
import ctypes

import numpy as np
import pytest

import layer_reference as ref


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


def off(p, by):
    return ctypes.c_void_p(p.value + by)


def caller(f, names, ok):
    names = names.split()
    assert len(names) == len(ok)
    return lambda **kw: f(*[kw.get(name, v) for name, v in zip(names, ok)])


def test_quantize_and_decode_refusals(qnn, p):
    call = caller(qnn.lib.qnn_i8_quantize, "x type rows width ldx codes ldc scales stream", (p, 1, 4, 40, 40, p, 48, p, None))
    for bad in ({"x": None}, {"codes": None}, {"scales": None}, {"type": 3}, {"type": -1}, {"rows": -1}, {"width": 0}, {"ldx": 39}, {"ldc": 32}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"codes": off(p, 8)}, {"ldc": 40}, {"ldc": 50}, {"x": off(p, 1)}, {"type": 0, "x": off(p, 2)}, {"scales": off(p, 2)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(width=131073, ldx=131073, ldc=131088) == qnn.E_RANGE and call(rows=1 << 31) == qnn.E_RANGE
    assert call(rows=0) == qnn.OK and call(rows=0, x=None, codes=None, scales=None) == qnn.OK
    call = caller(qnn.lib.qnn_i8_decode, "codes scales rows width ldc type out ldo stream", (p, p, 4, 40, 48, 1, p, 40, None))
    for bad in ({"codes": None}, {"scales": None}, {"out": None}, {"type": 9}, {"rows": -1}, {"width": 0}, {"ldc": 32}, {"ldo": 39}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"codes": off(p, 1)}, {"ldc": 41}, {"out": off(p, 1)}, {"scales": off(p, 1)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(rows=0, codes=None, out=None) == qnn.OK


def test_gemm_refusals_and_plan(qnn, p):
    call = caller(qnn.lib.qnn_i8_gemm, "x xs rows ldx w ws n k ldw bias type y ldy stream", (p, p, 4, 48, p, p, 8, 40, 48, None, 1, p, 8, None))
    for bad in ({"x": None}, {"xs": None}, {"w": None}, {"ws": None}, {"y": None}, {"type": 5}, {"rows": -1}, {"n": 0}, {"k": 0}, {"k": -3},
                {"ldx": 32}, {"ldw": 32}, {"ldy": 7}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"x": off(p, 4)}, {"w": off(p, 8)}, {"ldx": 40}, {"ldw": 41}, {"xs": off(p, 2)}, {"ws": off(p, 1)}, {"bias": off(p, 2)}, {"y": off(p, 1)},
                {"type": 0, "y": off(p, 2)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    for bad in ({"k": 131072, "ldx": 131072, "ldw": 131072}, {"n": 65535 * 16 + 1, "ldy": 65535 * 16 + 1}, {"rows": 1 << 23}):
        assert call(**bad) == qnn.E_RANGE, bad
    assert call(rows=0) == qnn.OK and call(rows=0, x=None, xs=None, y=None) == qnn.OK and call(rows=0, w=None) == qnn.E_ARG
    tile, ranks = ctypes.c_int(), ctypes.c_int()
    f = qnn.lib.qnn_i8_plan
    assert f(0, 8, 8, ctypes.byref(tile), ctypes.byref(ranks)) == qnn.E_ARG and f(1, 8, 8, None, ctypes.byref(ranks)) == qnn.E_ARG
    assert f(1, 8, 131072, ctypes.byref(tile), ctypes.byref(ranks)) == qnn.E_RANGE
    for rows, n, k in [(1, 64, 1), (1, 8192, 8192), (16, 128, 100), (33, 4096, 4096), (100, 300, 200), (8192, 8192, 8192), (1 << 20, 128, 64), ((1 << 23) - 1, 16, 16), ((1 << 23) - 1, 1, 131071), (1 << 21, 65535 * 16, 1)]:
        tile, ranks = qnn.i8_plan(rows, n, k)
        assert tile in (16, 32, 64, 128, 256) and ranks in (0, 1, 2, 4, 8) and ranks <= -(-k // 128)      # every rank has a step
        assert ranks == 0 or -(-rows // tile) <= 65535
    assert qnn.i8_plan(8192, 8192, 8192)[1] == 0 and qnn.i8_plan(1, 8192, 8192)[0] == 16


def test_norm_refusals(qnn, p):
    call = caller(qnn.lib.qnn_rms_norm, "x type rows width ldx residual ldr gain gain_type eps h ldh y ldy codes ldc scales rstd stream",
                  (p, 1, 4, 40, 40, p, 40, p, 1, 1e-6, p, 40, p, 40, p, 48, p, p, None))
    for bad in ({"x": None}, {"gain": None}, {"h": None}, {"y": None, "codes": None}, {"scales": None}, {"type": 3}, {"gain_type": 2}, {"gain_type": 7},
                {"rows": -1}, {"width": 0}, {"ldx": 39}, {"ldr": 39}, {"ldh": 39}, {"ldy": 39}, {"ldc": 32}, {"eps": -1.0}, {"eps": float("nan")},
                {"eps": float("inf")}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"x": off(p, 1)}, {"residual": off(p, 1)}, {"h": off(p, 1)}, {"y": off(p, 1)}, {"codes": off(p, 4)}, {"ldc": 44}, {"gain": off(p, 1)},
                {"gain_type": 0, "gain": off(p, 2)}, {"rstd": off(p, 2)}, {"scales": off(p, 1)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(width=32769, ldx=32769) == qnn.E_RANGE and call(rows=1 << 31) == qnn.E_RANGE
    assert call(rows=0) == qnn.OK and call(rows=0, x=None, y=None, codes=None, h=None) == qnn.OK and call(rows=0, gain=None) == qnn.E_ARG
    f = qnn.lib.qnn_rms_norm_backward_workspace
    assert f(0, 40) == 0 and f(4, 0) == 0 and f(4, 32769) == 0 and f(1, 40) >= 160 and f(10 ** 6, 4096) % 256 == 0
    need = f(4, 40)
    call = caller(qnn.lib.qnn_rms_norm_backward, "dy type rows width lddy h ldh gain gain_type rstd dh lddh dx lddx dgain ws ws_bytes stream",
                  (p, 1, 4, 40, 40, p, 40, p, 0, p, p, 40, p, 40, p, p, need, None))
    for bad in ({"dy": None}, {"h": None}, {"gain": None}, {"rstd": None}, {"dx": None}, {"dgain": None}, {"ws": None}, {"ws_bytes": need - 1},
                {"type": 4}, {"gain_type": 2}, {"rows": -1}, {"width": 0}, {"lddy": 39}, {"ldh": 39}, {"lddh": 39}, {"lddx": 39}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"dy": off(p, 1)}, {"h": off(p, 1)}, {"dh": off(p, 1)}, {"dx": off(p, 1)}, {"dgain": off(p, 2)}, {"rstd": off(p, 2)}, {"ws": off(p, 16)}):
        assert call(**bad) == qnn.E_ALIGN, bad


def test_route_refusals(qnn, p):
    f = qnn.lib.qnn_route_workspace
    assert f(0, 8, 2) == 0 and f(10, 8, 2) == 0 and f(10, 8, 9) == 0 and f(10, 1025, 2) == 0 and f(10 ** 6, 64, 33) == 0 and f(1 << 29, 8, 2) == 0
    need = f(5000, 64, 4)
    assert need > 0 and need % 256 == 0
    call = caller(qnn.lib.qnn_route, "logits type tokens experts ld top flags bias groups top_groups factor mask chosen weights order place offsets ws ws_bytes stream",
                  (p, 0, 5000, 64, 64, 4, 7, p, 8, 4, 1.0, p, p, p, p, p, p, p, need, None))
    for bad in ({"logits": None}, {"chosen": None}, {"weights": None}, {"order": None}, {"place": None}, {"offsets": None}, {"ws": None}, {"ws_bytes": need - 1},
                {"type": 3}, {"tokens": -1}, {"experts": 0}, {"experts": 1025, "ld": 1025, "groups": 1, "top_groups": 1}, {"ld": 63}, {"top": 0}, {"top": 33},
                {"top": 65}, {"flags": 8}, {"groups": 0}, {"groups": 7}, {"groups": 64}, {"top_groups": 0}, {"top_groups": 9}, {"top": 17, "top_groups": 2},
                {"experts": 8, "top_groups": 8, "ld": 8}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"logits": off(p, 2)}, {"bias": off(p, 1)}, {"chosen": off(p, 2)}, {"weights": off(p, 2)}, {"order": off(p, 1)}, {"place": off(p, 1)},
                {"offsets": off(p, 2)}, {"ws": off(p, 128)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(factor=float("inf")) == qnn.E_SCALE and call(factor=float("nan")) == qnn.E_SCALE
    assert call(tokens=1 << 28) == qnn.E_RANGE
    assert call(tokens=0, offsets=None, order=None, place=None) == qnn.OK
    call = caller(qnn.lib.qnn_route_backward, "dw logits type tokens experts ld top flags chosen factor out ldd stream",
                  (p, p, 0, 5, 64, 64, 4, 3, p, 1.0, p, 64, None))
    for bad in ({"dw": None}, {"logits": None}, {"chosen": None}, {"out": None}, {"type": 3}, {"tokens": -1}, {"experts": 0}, {"top": 65}, {"top": 0},
                {"flags": 8}, {"ld": 63}, {"ldd": 63}):
        assert call(**bad) == qnn.E_ARG, bad
    for bad in ({"dw": off(p, 2)}, {"logits": off(p, 2)}, {"chosen": off(p, 2)}, {"out": off(p, 2)}):
        assert call(**bad) == qnn.E_ALIGN, bad
    assert call(factor=float("nan")) == qnn.E_SCALE and call(tokens=1 << 28) == qnn.E_RANGE and call(tokens=0) == qnn.OK


# ------------------------------------------------------------------------------------------------ the plain forms, by hand

def test_plain_quantize():
    codes, scales = ref.quantize(np.array([[127.0, -0.5, 1.5, 2.5], [0, 0, 0, 0], [np.inf, 1, 1, 1]], dtype=np.float32))
    assert codes.tolist() == [[127, 0, 2, 2], [0] * 4, [0] * 4] and scales[0] == 1 and scales[1] == 2.0 ** -126 and np.isnan(scales[2])


def test_plain_route():
    l = np.array([[0.0, np.log(2.0), np.log(3.0), -np.inf], [5.0, 5.0, 1.0, 5.0]])
    chosen, w, order, place, offsets = ref.route(l, 2, renormalise=False)
    assert chosen.tolist() == [[2, 1], [0, 1]] and np.allclose(w[0], [3 / 6, 2 / 6])
    assert offsets.tolist() == [0, 1, 3, 4, 4] and order.tolist() == [2, 1, 3, 0] and place.tolist() == [[3, 1], [0, 2]]
    assert np.allclose(ref.route(l, 2)[1][0], [0.6, 0.4])
    # a bias moves the choice and not the weights; groups 0 (experts 0, 1) and 1 (2, 3)
    chosen, w, *_ = ref.route(l, 1, bias=np.array([1.0, 0, 0, 0]), renormalise=False)
    assert chosen.tolist() == [[0], [0]] and np.isclose(w[0, 0], 1 / 6)
    assert ref.route(l, 2, groups=2, top_groups=1)[0].tolist() == [[2, -1], [0, 1]]
    assert ref.route(l, 2, groups=2, top_groups=1, group_score="top2")[0].tolist() == [[1, 0], [0, 1]]
    chosen, w, order, *_ = ref.route(l, 2, mask=np.array([False, True]))
    assert chosen.tolist() == [[-1, -1], [0, 1]] and w[0].tolist() == [0, 0] and order.tolist() == [2, 3, -1, -1]


def test_plain_backward_forms_against_differences():
    rng = np.random.default_rng(0)
    h, gain, c, d = rng.standard_normal((2, 9)), rng.standard_normal(9), rng.standard_normal((2, 9)), rng.standard_normal((2, 9))
    f = lambda h, g: (ref.norm(h, g, 1e-3)[0] * c).sum() + (h * d).sum()
    dx, dgain = ref.norm_backward(c, h, gain, ref.norm(h, gain, 1e-3)[1], d)
    for at in np.ndindex(2, 9):
        s = np.zeros((2, 9))
        s[at] = 1e-6
        assert abs((f(h + s, gain) - f(h - s, gain)) / 2e-6 - dx[at]) < 1e-6
    for i in range(9):
        s = np.zeros(9)
        s[i] = 1e-6
        assert abs((f(h, gain + s) - f(h, gain - s)) / 2e-6 - dgain[i]) < 1e-6

"""Root-mean-square norm with a residual, real and in 8 bits, and its backward products, against 64 bits (layer_reference)."""
import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def real(t, rng, shape, dtype, size=1.0):
    v = t.from_numpy((rng.standard_normal(shape) * size).astype(np.float32)).to(ref.torch_type(dtype))
    return v.to(DEV)


def wide(x):
    return x.cpu().double().numpy()


def check(got, want, bound):
    got = wide(got)
    assert got.shape == want.shape and np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)


def check_norm(t, qnn, x, gain, residual, dtype):
    y, h, rstd = qnn.rms_norm(x, gain, EPS, residual)
    if residual is None:
        assert h is x
    else:
        assert t.equal(h, (x.float() + residual.float()).to(x.dtype))
    want, r = ref.norm(wide(h), wide(gain), EPS)
    check(rstd, r, r * ref.RSTD_ROUNDINGS * ref.U32)
    off = np.abs(want) * ref.Y_ROUNDINGS * ref.U32
    check(y, want, off + ref.rounding(np.abs(want) + off, dtype))
    rows, y2, h2, rstd2 = qnn.rms_norm_i8(x, gain, EPS, residual, both=True)
    assert t.equal(y2, y) and t.equal(h2, h) and t.equal(rstd2, rstd)
    alone, h3, rstd3 = qnn.rms_norm_i8(x, gain, EPS, residual)
    assert t.equal(alone.codes, rows.codes) and t.equal(alone.scales, rows.scales) and t.equal(rstd3, rstd)
    scales, codes = wide(rows.scales), wide(rows.codes)
    most = np.maximum(np.max(np.abs(want), axis=1) / 127, 2.0 ** -126)
    assert np.all(np.abs(scales - most) <= most * (ref.Y_ROUNDINGS + 1) * ref.U32)
    # a code is the nearest, but for quotients that lie next to a half: off by the roundings of y and scale, times 127
    assert np.all(np.abs(codes * scales[:, None] - want) <= scales[:, None] * (0.5 + 127 * (2 * ref.Y_ROUNDINGS + 4) * ref.U32))
    assert np.all(np.max(np.abs(codes), axis=1) == np.where(np.max(np.abs(want), axis=1) > 0, 127, 0))


SIZES = [(1, 1), (1, 8), (3, 64), (5, 100), (2, 256), (7, 264), (3, 1001), (300, 512), (1, 4096), (297, 2048), (2, 8192), (3, 8200), (1, 16384), (2, 16383),
         (400, 333), (5, 1538), (3, 16400), (2, 32768), (2, 32767)]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm(t, qnn, dtype, rows, width):
    rng = np.random.default_rng(rows * 31 + width)
    x, residual = real(t, rng, (rows, width), dtype, 2.0), real(t, rng, (rows, width), dtype)
    gain = (1 + 0.3 * t.randn(width, device=DEV, generator=t.Generator(device=DEV).manual_seed(width))).to(x.dtype)
    check_norm(t, qnn, x, gain, residual, dtype)
    check_norm(t, qnn, x, gain, None, dtype)
    check_norm(t, qnn, x, gain.float() * 1.001, residual, dtype)                  # a gain in fp32


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_norm_strides(t, qnn, dtype):
    rng = np.random.default_rng(2)
    big, other = real(t, rng, (6, 700), dtype), real(t, rng, (6, 900), dtype)
    for at, width in ((0, 512), (1, 512), (8, 640), (13, 333)):
        gain = real(t, rng, width + 1, dtype)[1:]                                 # starts off 16 bytes
        check_norm(t, qnn, big[:, at:at + width], gain, other[:, 8:8 + width], dtype)
        check_norm(t, qnn, big[:, at:at + width], gain.clone(), other[:, 8:8 + width], dtype)


@pytest.mark.parametrize("width", [256, 257])
def test_norm_special_values(t, qnn, width):
    """Rows of zeros, tiny ones, infinities, NaN, and a gain that is not finite."""
    x = t.ones((6, width), device=DEV)
    x[1] = 0
    x[2] = 1e-25
    x[3, width - 1] = float("inf")
    x[4, 3] = float("nan")
    gain = t.ones(width, device=DEV)
    y, _, rstd = qnn.rms_norm(x, gain, EPS)
    assert bool((y[1] == 0).all()) and bool((rstd[3] == 0)) and bool(y[3, width - 1].isnan()) and bool(y[4].isnan().all())
    assert np.allclose(wide(y[2]), 1e-25 / np.sqrt(EPS), rtol=1e-6) and not bool(y[5].isnan().any())
    rows, _, _ = qnn.rms_norm_i8(x, gain, EPS)
    assert rows.scales.isnan().tolist() == [False, False, False, True, True, False] and bool((rows.codes[3:5] == 0).all())
    assert rows.scales[1].item() == 2.0 ** -126 and bool((rows.codes[2] == 127).all())
    gain[7] = float("nan")
    assert bool(qnn.rms_norm_i8(x, gain, EPS)[0].scales.isnan().all())
    assert bool(qnn.rms_norm(x[:1], gain, EPS)[0].isnan()[0, 7]) and qnn.rms_norm(x[:1], gain, EPS)[0].isnan().sum().item() == 1


@pytest.mark.parametrize("width", [1024, 1001])
def test_norm_in_place(t, qnn, width):
    """The C call with h over x, over the residual, and y over x."""
    import ctypes as C
    x, r, gain = (t.randn((5, width), device=DEV) for _ in range(3))
    gain = gain[0].contiguous()
    y, h, _ = qnn.rms_norm(x, gain, EPS, r)
    plain, _, _ = qnn.rms_norm(x, gain, EPS)
    p = lambda v: C.c_void_p(v.data_ptr())
    stream = C.c_void_p(t.cuda.current_stream().cuda_stream)
    for over in ("x", "r"):
        a, b, out = x.clone(), r.clone(), t.empty_like(x)
        target = a if over == "x" else b
        assert qnn.lib.qnn_rms_norm(p(a), 0, 5, width, width, p(b), width, p(gain), 0, EPS, p(target), width, p(out), width, None, 0, None, None, stream) == 0
        assert t.equal(target, h) and t.equal(out, y)
    a = x.clone()
    assert qnn.lib.qnn_rms_norm(p(a), 0, 5, width, width, None, 0, p(gain), 0, EPS, None, 0, p(a), width, None, 0, None, None, stream) == 0
    assert t.equal(a, plain)


# ------------------------------------------------------------------------------------------------ backward

@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", SIZES + [(1000, 72), (593, 1000)])
def test_backward(t, qnn, dtype, rows, width):
    rng = np.random.default_rng(rows + width)
    h, dy, dh = real(t, rng, (rows, width), dtype, 2.0), real(t, rng, (rows, width), dtype, 0.3), real(t, rng, (rows, width), dtype)
    for gain in (real(t, rng, width, dtype), real(t, rng, width, "fp32")):
        rstd = t.from_numpy(ref.norm(wide(h), wide(gain), EPS)[1].astype(np.float32)).to(DEV)
        for other in (None, dh):
            dx, dgain = qnn.rms_norm_backward(dy, h, gain, rstd, other)
            args = (wide(dy), wide(h), wide(gain), wide(rstd), None if other is None else wide(other))
            want, wgain = ref.norm_backward(*args)
            bx, bg = ref.norm_backward_bounds(*args, dtype)
            check(dx, want, bx)
            check(dgain, wgain, bg + 1e-30)
            again = qnn.rms_norm_backward(dy, h, gain, rstd, other)
            assert t.equal(again[0], dx) and t.equal(again[1], dgain)


def test_backward_against_differences(t, qnn):
    """The gradient of sum(y * c) + sum(h * d) with respect to x and gain, by central differences in 64 bits."""
    rng = np.random.default_rng(3)
    rows, width = 3, 40
    x, c, d = (rng.standard_normal((rows, width)).astype(np.float32) for _ in range(3))
    gain = (1 + 0.2 * rng.standard_normal(width)).astype(np.float32)
    f = lambda x, g: (ref.norm(x, g, EPS)[0] * c).sum() + (x * d).sum()
    on = lambda v: t.from_numpy(v).to(DEV)
    _, _, rstd = qnn.rms_norm(on(x), on(gain), EPS)
    dx, dgain = (wide(v) for v in qnn.rms_norm_backward(on(c), on(x), on(gain), rstd, on(d)))
    x64, g64, e = x.astype(np.float64), gain.astype(np.float64), 1e-5
    for r in range(rows):
        for i in range(0, width, 7):
            s = np.zeros_like(x64)
            s[r, i] = e
            assert abs((f(x64 + s, g64) - f(x64 - s, g64)) / (2 * e) - dx[r, i]) < 1e-5 * (1 + abs(dx[r, i]))
    for i in range(width):
        s = np.zeros_like(g64)
        s[i] = e
        assert abs((f(x64, g64 + s) - f(x64, g64 - s)) / (2 * e) - dgain[i]) < 1e-5 * (1 + abs(dgain[i]))


def test_backward_strides_and_no_rows(t, qnn):
    rng = np.random.default_rng(4)
    for at, width in ((0, 512), (3, 512), (8, 333)):
        big = [real(t, rng, (70, 700), "bf16") for _ in range(3)]
        gain, rstd = real(t, rng, width, "bf16"), t.rand(70, device=DEV)
        cut = [b[:, at:at + width] for b in big]
        dx, dgain = qnn.rms_norm_backward(cut[0], cut[1], gain, rstd, cut[2])
        dx2, dgain2 = qnn.rms_norm_backward(*(c.contiguous() for c in cut[:2]), gain, rstd, cut[2].contiguous())
        args = (wide(cut[0]), wide(cut[1]), wide(gain), wide(rstd), wide(cut[2]))
        bx, bg = ref.norm_backward_bounds(*args, "bf16")
        check(dx, ref.norm_backward(*args)[0], bx)
        check(dx2, ref.norm_backward(*args)[0], bx)
        check(dgain, wide(dgain2), 2 * bg)
    empty = t.zeros((0, 16), device=DEV)
    dx, dgain = qnn.rms_norm_backward(empty, empty, t.ones(16, device=DEV), t.zeros(0, device=DEV))
    assert dx.shape == (0, 16) and bool((dgain == 0).all())
    y, h, rstd = qnn.rms_norm(empty, t.ones(16, device=DEV))
    assert y.shape == (0, 16) and rstd.shape == (0,)


def test_captured(t, qnn):
    x, r, gain = (t.randn((40, 1024), device=DEV).bfloat16() for _ in range(3))
    gain = gain[0].contiguous()
    def step():
        rows, y, h, rstd = qnn.rms_norm_i8(x, gain, EPS, r, both=True)
        return (rows.codes, rows.scales, y, h) + qnn.rms_norm_backward(y, h, gain, rstd, x)
    step()
    t.cuda.synchronize()
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        out = step()
    for _ in range(3):
        x.normal_()
        r.normal_()
        g.replay()
        for a, b in zip(out, step()):
            assert t.equal(a, b)


def test_refusals(t, qnn):
    x, gain = t.randn((4, 40), device=DEV), t.ones(40, device=DEV)
    rstd = t.ones(4, device=DEV)
    for bad in (lambda: qnn.rms_norm(x, gain[:39]), lambda: qnn.rms_norm(x, gain.bfloat16()), lambda: qnn.rms_norm(x, gain, residual=x.bfloat16()),
                lambda: qnn.rms_norm(x, gain, residual=x[:3]), lambda: qnn.rms_norm(x.t(), gain), lambda: qnn.rms_norm(x, gain.cpu()),
                lambda: qnn.rms_norm(x.clone().requires_grad_(), gain), lambda: qnn.rms_norm(x, gain.clone().requires_grad_()),
                lambda: qnn.rms_norm_backward(x, x[:3], gain, rstd), lambda: qnn.rms_norm_backward(x, x, gain, rstd[:3]),
                lambda: qnn.rms_norm_backward(x, x, gain, rstd.double()), lambda: qnn.rms_norm_backward(x, x, gain, rstd, x.bfloat16()),
                lambda: qnn.rms_norm_backward(x, x, gain, None)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qnn.rms_norm(x, gain, -1.0), lambda: qnn.rms_norm(x, gain, float("nan")),
                lambda: qnn.rms_norm(t.zeros((1, 32769), device=DEV), t.ones(32769, device=DEV)),
                lambda: qnn.rms_norm_backward(x, x, gain, rstd, workspace=t.zeros(8, dtype=t.uint8, device=DEV))):
        with pytest.raises(qnn.QnnError):
            bad()

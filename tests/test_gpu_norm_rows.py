"""A row's norm, codes and gradient do not depend on the rows beside it: alone, in a short call and in a long one, bit for bit."""
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("width", [8, 128, 136, 256, 264, 384, 504, 512, 520, 1000, 1024, 2040, 2048, 3000, 4096, 4104, 8192, 16384, 17, 333, 1001, 5000])
def test_rows_do_not_depend_on_one_another(t, qnn, dtype, width):
    g = t.Generator(device=DEV).manual_seed(width)
    real = lambda *shape: t.randn(shape, device=DEV, generator=g).to(ref.torch_type(dtype))
    x, r, dy, gain = real(600, width), real(600, width), real(600, width), 1 + 0.2 * real(width)
    rows, y, h, rstd = qnn.rms_norm_i8(x, gain, EPS, r, both=True)
    dx, _ = qnn.rms_norm_backward(dy, h, gain, rstd, x)
    codes, scales = qnn.i8_quantize(x)
    for some in ((0, 1), (299, 300), (597, 600), (100, 396), (50, 347), (0, 599)):
        a, b = some
        rows1, y1, h1, rstd1 = qnn.rms_norm_i8(x[a:b], gain, EPS, r[a:b], both=True)
        for one, all_ in ((rows1.codes, rows.codes), (rows1.scales, rows.scales), (y1, y), (h1, h), (rstd1, rstd)):
            assert t.equal(one, all_[a:b])
        assert t.equal(qnn.rms_norm_backward(dy[a:b], h[a:b], gain, rstd[a:b], x[a:b])[0], dx[a:b])
        assert t.equal(qnn.i8_quantize(x[a:b]).codes, codes[a:b])

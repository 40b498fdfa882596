"""The codes of the norm and of the quantiser: one rule, operation for operation in fp32 (layer_reference.quantize), also where quotients
lie next to a half."""
import numpy as np
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


# one for each kernel: packs of 1, 2, 4 and 8 a thread, one warp a row, element by element, and rows read twice
SIZES = [(5, 64), (5, 4096), (300, 4096), (4, 8192), (3, 12000), (3, 16384), (5, 100), (4, 1001), (3, 8191), (2, 16381), (2, 32768), (2, 32767)]


def halves(rng, rows, width):
    """Rows whose quotients are halves, as nearly as fp32 has them: (k + 1/2) of a step and one element of 127 of them."""
    k = rng.integers(-127, 127, (rows, width)) + 0.5
    k[:, width // 2] = 127.0
    return (k * rng.uniform(0.5, 2.0, (rows, 1))).astype(np.float32)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm_codes_follow_the_rule(t, qnn, dtype, rows, width):
    """y as the call computes it, in fp32 from the rstd that it returns: (h * gain) * rstd; its codes and scales bit for bit."""
    rng = np.random.default_rng(rows + width)
    kind = ref.torch_type(dtype)
    for x, gain in ((halves(rng, rows, width), np.ones(width, dtype=np.float32)),
                    (rng.standard_normal((rows, width)).astype(np.float32), (1 + 0.2 * rng.standard_normal(width)).astype(np.float32))):
        x, gain = t.from_numpy(x).to(kind).to(DEV), t.from_numpy(gain).to(DEV)
        for g in (gain, gain.to(kind)):
            got, y, h, rstd = qnn.rms_norm_i8(x, g, EPS, both=True)
            y32 = (h.float().cpu().numpy() * g.float().cpu().numpy()) * rstd.cpu().numpy()[:, None]
            assert y32.dtype == np.float32 and t.equal(y.cpu(), t.from_numpy(y32).to(kind))
            codes, scales = ref.quantize(y32)
            assert np.array_equal(got.scales.cpu().numpy(), scales)
            assert np.array_equal(got.codes.cpu().numpy(), codes)
            if dtype == "fp32":                                       # the quantiser of the same numbers gives the same
                again = qnn.i8_quantize(y)
                assert t.equal(again.codes, got.codes) and t.equal(again.scales, got.scales)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,width", SIZES + [(2, 40000), (2, 40001)])
def test_quantiser_next_to_halves(t, qnn, dtype, rows, width):
    x = t.from_numpy(halves(np.random.default_rng(rows * width), rows, width)).to(ref.torch_type(dtype))
    got = qnn.i8_quantize(x.to(DEV))
    codes, scales = ref.quantize(x.float().numpy())
    assert np.array_equal(got.scales.cpu().numpy(), scales) and np.array_equal(got.codes.cpu().numpy(), codes)


def borders():
    """(y, S) whose quotients lie next to half a step of fp32 off a half: with m the exponent of the half h / 2, y = (S * h + d) / 2 and S within
    a few units of d * 2^(23 - m), y / S is off that border by j / 2S steps, a whole j."""
    for m in range(-1, 7):
        for d in range(1, 2 ** (m + 2) + 2):
            for j in range(-4, 5):
                s = d * 2 ** (23 - m) + j
                if not 2 ** 23 <= s < 2 ** 24:
                    continue
                for h in range(max(1, 2 ** (m + 1) | 1), 2 ** (m + 2), 2):
                    for y2 in (s * h + d, s * h - d):
                        y = np.float32(y2 / 2)
                        if int(2 * float(y)) == y2 and h < 254:
                            yield y, s


@pytest.mark.parametrize("exponent", [-149, -126, -100, -83, -60, -23, 0, 60, 97])
def test_quotients_next_to_a_border(t, qnn, exponent):
    cases = np.array(list(borders()))
    y, s = (cases * 2.0 ** exponent).astype(np.float32).T
    # a row's largest number, chosen so that its 127th rounds to the scale
    step = np.spacing((s * np.float32(127)).astype(np.float32))
    most = np.stack([s * np.float32(127) + k * step for k in range(-2, 3)]).astype(np.float32)
    fits = (most / np.float32(127)).astype(np.float32) == s
    most = np.take_along_axis(most, np.argmax(fits, axis=0)[None], 0)[0]
    assert len(y) > 700 and fits.any(axis=0).all()
    for width in (32, 33):
        x = np.zeros((len(y), width), dtype=np.float32)
        x[:, 0], x[:, 5], x[:, width - 1] = most, y, -y
        codes, scales = ref.quantize(x)
        assert np.array_equal(scales, s)
        # (these are cases that the product with the inverse decides otherwise)
        assert (np.rint(y.astype(np.float64) * (np.float32(1) / s).astype(np.float64)) != codes[:, 5]).sum() > 150
        got = qnn.i8_quantize(t.from_numpy(x).to(DEV))
        assert np.array_equal(got.scales.cpu().numpy(), scales) and np.array_equal(got.codes.cpu().numpy(), codes)

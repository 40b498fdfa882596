"""Rows in 8 bits on the GPU: codes and scales, decoding, and their products, each bit for bit as the definition's operations give them."""
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


def rows_of(t, qnn, codes, scales):
    """Codes in an array whose rows start on 16 bytes."""
    n, k = codes.shape
    full = t.full((n, (k + 15) // 16 * 16), 77, dtype=t.int8, device=DEV)      # what lies behind a row is not read
    full[:, :k] = t.from_numpy(codes).to(DEV)
    return qnn.I8Rows(full[:, :k], t.from_numpy(scales).to(DEV))


def random_rows(rng, n, k, low=-127):
    return rng.integers(low, 128, size=(n, k)).astype(np.int8), (rng.uniform(0.5, 1.5, n) * 0.01).astype(np.float32)


def same(t, got, want):
    got = got.cpu()
    nan = want.isnan()
    assert got.dtype == want.dtype and got.shape == want.shape
    assert t.equal(got.isnan(), nan) and t.equal(got[~nan], want[~nan])


# ------------------------------------------------------------------------------------------------ codes

@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 7), (3, 8), (5, 64), (4, 255), (2, 256), (9, 264), (7, 1000), (3, 1001), (2, 4096), (1, 8192),
                                    (2, 8200), (400, 1032), (300, 129), (1, 16384), (2, 16383), (3, 16400), (2, 28672), (2, 28671), (1, 40000), (2, 131072), (1, 131071)])
def test_quantize_and_decode(t, qnn, dtype, rows, k):
    rng = np.random.default_rng(rows * 7919 + k)
    x = t.from_numpy((rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1)) * 3)).astype(np.float32)).to(ref.torch_type(dtype)).to(DEV)
    got = qnn.i8_quantize(x)
    codes, scales = ref.quantize(x.float().cpu().numpy())
    assert got.codes.stride(0) % 16 == 0 and np.array_equal(got.scales.cpu().numpy(), scales, equal_nan=True)      # (fp16: rows with infinities)
    assert np.array_equal(got.codes.cpu().numpy(), codes)
    for kind in ref.TYPES:
        want = t.from_numpy(codes.astype(np.float32) * scales[:, None]).to(ref.torch_type(kind))
        same(t, qnn.i8_decode(got, ref.torch_type(kind)), want)


@pytest.mark.parametrize("k", [256, 257])
def test_quantize_special_values(t, qnn, k):
    """Zeros, values below the smallest scale, quotients half-way between codes, infinities and NaN, one of them at the end."""
    x = t.zeros((9, k))
    x[1] = 1e-40
    x[2, 0], x[2, 1] = 127.0, -0.5
    x[2, 2:129] = t.arange(127) + 0.5
    x[3, 0], x[3, k - 1] = 3.0, float("inf")
    x[4, 5] = float("nan")
    x[5, k - 1] = -float("inf")
    x[6, 0], x[6, 1] = 3.0e38, -1.5e38
    x[7, k - 1] = -2.0 ** -126 * 127
    x[8] = -t.linspace(0, 127, k)
    got = qnn.i8_quantize(x.to(DEV))
    codes, scales = ref.quantize(x.numpy())
    assert np.array_equal(got.scales.cpu().numpy(), scales, equal_nan=True) and np.array_equal(got.codes.cpu().numpy(), codes)
    back = qnn.i8_decode(got, t.float32).cpu()
    assert bool(back[3:6].isnan().all()) and bool((back[:2] == 0).all()) and not bool(back[6:].isnan().any())
    y = qnn.i8_gemm(got, got, t.float32).cpu()                    # products with such a row are NaN, the others are not
    bad = t.tensor([False, False, False, True, True, True, False, False, False])
    assert t.equal(y.isnan(), bad.view(-1, 1) | bad.view(1, -1))


def test_quantize_strided_rows(t, qnn):
    for kind in ref.TYPES:
        big = t.randn((6, 700), device=DEV).to(ref.torch_type(kind))
        for at, k in ((0, 512), (1, 512), (8, 640), (13, 333)):
            got = qnn.i8_quantize(big[:, at:at + k])
            codes, scales = ref.quantize(big[:, at:at + k].float().cpu().numpy())
            assert np.array_equal(got.codes.cpu().numpy(), codes) and np.array_equal(got.scales.cpu().numpy(), scales)
            out = t.full((6, 800), 5.0, device=DEV, dtype=big.dtype)
            qnn.i8_decode(got, big.dtype, out=out[:, at:at + k])
            assert t.equal(out[:, at:at + k], qnn.i8_decode(got, big.dtype))
            assert bool((out[:, :at] == 5).all()) and bool((out[:, at + k:] == 5).all())


# ------------------------------------------------------------------------------------------------ products

SIZES = [(1, 1, 1), (1, 7, 3), (2, 128, 128), (3, 129, 255), (1, 257, 1000), (8, 64, 2049), (16, 300, 4096), (17, 130, 640), (31, 48, 264),
         (32, 1040, 136), (33, 200, 513), (64, 127, 1000), (65, 64, 96), (128, 384, 700), (129, 128, 512), (200, 777, 1001), (300, 1000, 130),
         (1, 40000, 256), (16, 16400, 128), (1, 64, 20000), (40, 16, 16384)]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_gemm(t, qnn, dtype, rows, n, k):
    rng = np.random.default_rng(rows * 1000003 + n * 1009 + k)
    (x, sx), (w, sw) = random_rows(rng, rows, k), random_rows(rng, n, k)
    bias = rng.standard_normal(n).astype(np.float32) if (rows + n + k) % 2 else None
    got = qnn.i8_gemm(rows_of(t, qnn, x, sx), rows_of(t, qnn, w, sw), ref.torch_type(dtype), None if bias is None else t.from_numpy(bias).to(DEV))
    same(t, got, ref.gemm(x, sx, w, sw, bias, dtype))
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,n,k", [(2100, 2300, 96), (2049, 2305, 257), (257, 19001, 130), (19000, 200, 64), (4000, 1500, 1000)])
def test_gemm_by_pairs(t, qnn, dtype, rows, n, k):
    """Sizes that the pairs of blocks serve: more tiles than pairs, edges of tiles in both directions, several bands of tokens."""
    assert qnn.i8_plan(rows, n, k)[1] == 0
    rng = np.random.default_rng(rows + n + k)
    (x, sx), (w, sw) = random_rows(rng, rows, k, -128), random_rows(rng, n, k, -128)
    bias = rng.standard_normal(n).astype(np.float32)
    xd, wd = rows_of(t, qnn, x, sx), rows_of(t, qnn, w, sw)
    got = qnn.i8_gemm(xd, wd, ref.torch_type(dtype), t.from_numpy(bias).to(DEV))
    # the whole sums by fp64 products on the GPU, which are exact below 2^53
    acc = t.from_numpy(x).to(DEV).double() @ t.from_numpy(w).to(DEV).double().t()
    want = acc.float() * xd.scales.view(-1, 1) * wd.scales + t.from_numpy(bias).to(DEV)
    assert t.equal(got, want.to(got.dtype)) and qnn.tensor_path_status() == 0


FORMS = {(16, 1): (5, 16, 32), (16, 2): (474, 130, 1201), (16, 4): (1, 16, 390), (16, 8): (1, 17, 925), (32, 1): (2087, 138, 32),
         (32, 2): (566, 407, 2598), (32, 4): (482, 129, 1923), (32, 8): (251, 129, 3590), (64, 1): (2821, 276, 32), (64, 2): (1062, 390, 2984),
         (64, 4): (530, 405, 3052), (64, 8): (457, 134, 4873), (128, 1): (2504, 777, 161), (128, 2): (798, 949, 4004), (128, 4): (991, 411, 2959),
         (128, 8): (204, 811, 10283), (128, 0): (2064, 900, 45), (256, 0): (1703, 1294, 538)}


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_gemm_by_every_form(t, qnn, dtype, form):
    """Every tile and split that the plan can choose, at a small size that it serves; operands that grow out of one another on the way
    (a call's result feeds the next one's rows), queued without a wait."""
    rows, n, k = FORMS[form]
    assert qnn.i8_plan(rows, n, k) == form
    rng = np.random.default_rng(rows + n + k)
    xd, wd = rows_of(t, qnn, *random_rows(rng, rows, k)), rows_of(t, qnn, *random_rows(rng, n, k))
    kind = ref.torch_type(dtype)
    acc = xd.codes.double() @ wd.codes.double().t()
    want = (acc.float() * xd.scales.view(-1, 1) * wd.scales).to(kind)
    t.cuda.synchronize()
    for _ in range(3):
        got = qnn.i8_gemm(xd, wd, kind)
        chained = qnn.i8_quantize(got)
        assert t.equal(got, want) and t.equal(chained.codes, qnn.i8_quantize(want).codes)
    assert qnn.tensor_path_status() == 0


def test_gemm_extreme_codes(t, qnn):
    """The longest contraction of the largest codes: the sum is 2^31 - 2^14, rounded once."""
    k = 131071
    x = rows_of(t, qnn, np.full((2, k), -128, dtype=np.int8), np.ones(2, dtype=np.float32))
    got = qnn.i8_gemm(x, x, t.float32).cpu()
    assert bool((got == float(np.float32(128 * 128 * k))).all())


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows", [1, 5, 40, 200])
def test_gemm_strides(t, qnn, dtype, rows):
    """Operands with gaps between rows, a result in a column range (aligned and not) of a larger array; nothing around it is written."""
    rng = np.random.default_rng(rows)
    (x, sx), (w, sw) = random_rows(rng, rows, 300), random_rows(rng, 77, 300)
    big = t.zeros((rows, 512), dtype=t.int8, device=DEV)
    big[:, 32:332] = t.from_numpy(x).to(DEV)
    xd = qnn.I8Rows(big[:, 32:332], t.from_numpy(sx).to(DEV))
    want = ref.gemm(x, sx, w, sw, None, dtype)
    for at in (0, 3, 8):
        out = t.full((rows + 2, 96), 9.0, dtype=ref.torch_type(dtype), device=DEV)
        qnn.i8_gemm(xd, rows_of(t, qnn, w, sw), ref.torch_type(dtype), out=out[1:rows + 1, at:at + 77])
        assert t.equal(out[1:rows + 1, at:at + 77].cpu(), want)
        out[1:rows + 1, at:at + 77] = 9.0
        assert bool((out == 9.0).all())


def test_gemm_no_rows(t, qnn):
    w = qnn.i8_quantize(t.randn((20, 40), device=DEV))
    x = qnn.i8_quantize(t.randn((0, 40), device=DEV))
    assert qnn.i8_gemm(x, w).shape == (0, 20) and qnn.i8_decode(x).shape == (0, 40)


def test_gemm_captured_and_on_another_stream(t, qnn):
    """A captured call reads what its buffers hold at the replay; a call on another stream gives the same bits."""
    w = qnn.i8_quantize(t.randn((500, 1024), device=DEV))
    for rows in (1, 20, 150):
        x = t.randn((rows, 1024), device=DEV)
        s = t.cuda.Stream()
        s.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(s):
            qnn.i8_gemm(qnn.i8_quantize(x), w)
        t.cuda.current_stream().wait_stream(s)
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            y = qnn.i8_gemm(qnn.i8_quantize(x), w, t.float32)
        for _ in range(3):
            x.normal_()
            g.replay()
            want = qnn.i8_gemm(qnn.i8_quantize(x), w, t.float32)
            assert t.equal(y, want)
            t.cuda.synchronize()
            q = qnn.i8_quantize(x, stream=s)
            z = qnn.i8_gemm(q, w, t.float32, stream=s)
            s.synchronize()
            assert t.equal(z, want)


def test_refusals(t, qnn):
    x, w = qnn.i8_quantize(t.randn((4, 40), device=DEV)), qnn.i8_quantize(t.randn((6, 40), device=DEV))
    odd = t.zeros((4, 41), dtype=t.int8, device=DEV)[:, :40]                     # rows that do not start on 16 bytes
    with pytest.raises(qnn.QnnError):
        qnn.i8_gemm(qnn.I8Rows(odd, x.scales), w)
    for bad in (lambda: qnn.i8_gemm(x, qnn.i8_quantize(t.randn((6, 48), device=DEV))),
                lambda: qnn.i8_gemm(x, w, t.float64), lambda: qnn.i8_gemm(x, w, t.int8), lambda: qnn.i8_gemm(x, w, "bf16"),
                lambda: qnn.i8_gemm(x, w, bias=t.zeros(5, device=DEV)), lambda: qnn.i8_gemm(x, w, bias=t.zeros(6)),
                lambda: qnn.i8_gemm(x, w, out=t.zeros((4, 6), device=DEV)),
                lambda: qnn.i8_gemm(qnn.I8Rows(x.codes.float(), x.scales), w), lambda: qnn.i8_gemm(qnn.I8Rows(x.codes, x.scales[:3]), w),
                lambda: qnn.i8_gemm(qnn.I8Rows(x.codes.cpu(), x.scales), w), lambda: qnn.i8_gemm(qnn.I8Rows(x.codes.t(), x.scales), w),
                lambda: qnn.i8_quantize(t.randn(4, 40)), lambda: qnn.i8_quantize(t.randn((4, 40), device=DEV).double()),
                lambda: qnn.i8_quantize(t.randn((4, 40), device=DEV).t()), lambda: qnn.i8_quantize(t.randn((4, 40), device=DEV, requires_grad=True)),
                lambda: qnn.i8_gemm(x._replace(scales=x.scales.clone().requires_grad_()), w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(qnn.QnnError):
        qnn.i8_quantize(t.zeros((1, 131073), device=DEV))

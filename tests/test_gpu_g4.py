"""Group-scaled 4-bit weights on the GPU against the plain 64-bit forms of g4_reference: packing, few rows, rows grouped
by expert, and the two backward products.  Bounds: g4_reference.bound."""
import numpy as np
import pytest

import g4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


DEV = "cuda:0"


def handle(qnn, t, codes, scales, alpha, n, k, group):
    return qnn.G4Weights(t.from_numpy(codes).to(DEV), t.from_numpy(scales).to(DEV), t.from_numpy(alpha).to(DEV), n, k, group)


def real(t, rng, shape, dtype, size=1.0):
    """Random values of a type on the GPU, and the same values in 64 bits."""
    v = t.from_numpy((rng.standard_normal(shape) * size).astype(np.float32)).to(ref.torch_type(dtype))
    return v.to(DEV), v.to(t.float64).numpy()


def check(got, exact, magnitude, length, dtype):
    got = got.to("cpu").double().numpy()
    assert got.shape == exact.shape
    err, tol = np.abs(got - exact), ref.bound(exact, magnitude, length, dtype)
    assert np.all(err <= tol), f"worst {np.max(err / tol):.3g} of its bound"


def offsets_of(t, counts, lead=0):
    return t.tensor(np.concatenate([[lead], lead + np.cumsum(counts)]), dtype=t.int32, device=DEV)


def grouped(counts, lead, f):
    """Calls f(expert, first, last) for each expert's rows."""
    at = lead
    for e, c in enumerate(counts):
        if c:
            f(e, at, at + c)
        at += c


# ------------------------------------------------------------------------------------------------ packing

@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("experts,n,k", [(1, 1, 1), (2, 130, 129), (3, 64, 300), (1, 300, 64)])
def test_pack_matches_plain_form(t, qnn, dtype, group, experts, n, k):
    rng = np.random.default_rng(n * k + group)
    w, w64 = real(t, rng, (experts, n, k), dtype, 0.03)
    got = qnn.g4_pack_weights(w, group)
    for e in range(experts):
        tt, byte, alpha = ref.quantize(w64[e].astype(np.float32), group)
        codes, scales = ref.store(tt, byte, group)
        assert np.float32(got.alpha[e].item()) == alpha
        assert np.array_equal(got.scales[e].cpu().numpy(), scales)
        assert np.array_equal(got.codes[e].cpu().numpy(), codes)


def test_pack_special_values(t, qnn):
    """Zero matrices, zero groups, ties, NaN."""
    w = t.zeros((2, 4, 256), device=DEV)
    w[1, 0, :128] = t.linspace(-15, 15, 128)                      # includes values half-way between codes
    w[1, 0, 0], w[1, 0, 1] = 15.0 * 448, float("nan")
    w[1, 1, 5] = 15.0
    got = qnn.g4_pack_weights(w, 128)
    assert got.alpha[0].item() == 0.0 and got.alpha[1].item() == 1.0
    for e in range(2):
        tt, byte, alpha = ref.quantize(w[e].cpu().numpy(), 128)
        codes, scales = ref.store(tt, byte, 128)
        assert np.array_equal(got.codes[e].cpu().numpy(), codes) and np.array_equal(got.scales[e].cpu().numpy(), scales)
    x = t.randn((3, 256), device=DEV)
    zero = qnn.G4Weights(got.codes[:1], got.scales[:1], got.alpha[:1], 4, 256, 128)
    assert t.equal(qnn.g4_matvec(x, zero), t.zeros((3, 4), device=DEV))


# ------------------------------------------------------------------------------------------------ few rows

@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (1, 7, 3), (2, 128, 128), (3, 129, 255), (1, 257, 1000), (8, 64, 2049),
                                      (5, 16, 1032), (11, 200, 136), (17, 130, 640), (33, 48, 264), (1, 1040, 4096), (2, 16, 8200), (4, 300, 16384)])
def test_matvec(t, qnn, dtype, group, rows, n, k):
    rng = np.random.default_rng(rows * 1000003 + n * 1009 + k + group)
    codes, scales, alpha, dense = ref.random_weights(rng, 1, n, k, group)
    x, x64 = real(t, rng, (rows, k), dtype)
    y = qnn.g4_matvec(x, handle(qnn, t, codes, scales, alpha, n, k, group))
    check(y, x64 @ dense[0].T, np.abs(x64) @ np.abs(dense[0]).T, k, dtype)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_matvec_strides_and_alignment(t, qnn, dtype):
    """Rows with gaps, rows that start off a 16-byte boundary, results into a column range of a larger array."""
    rng = np.random.default_rng(5)
    n, k, rows = 77, 250, 6
    codes, scales, alpha, dense = ref.random_weights(rng, 1, n, k, 64)
    w = handle(qnn, t, codes, scales, alpha, n, k, 64)
    big, big64 = real(t, rng, (rows, 300), dtype)
    for at in (0, 1, 8, 31):
        out = t.full((rows, 100), float("nan"), dtype=big.dtype, device=DEV)
        got = qnn.g4_matvec(big[:, at:at + k], w, out=out[:, 3:3 + n])
        xs = big64[:, at:at + k]
        check(got, xs @ dense[0].T, np.abs(xs) @ np.abs(dense[0]).T, k, dtype)
        assert bool(out[:, :3].isnan().all()) and bool(out[:, 3 + n:].isnan().all())
    one = big[2:3, 5:5 + k]                                       # a single row, whatever its stride
    check(qnn.g4_matvec(one, w), big64[2:3, 5:5 + k] @ dense[0].T, np.abs(big64[2:3, 5:5 + k]) @ np.abs(dense[0]).T, k, dtype)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_matvec_special_values_stay_in_their_row(t, qnn, dtype):
    rng = np.random.default_rng(6)
    n, k, rows = 40, 300, 4
    t_codes = rng.integers(0, 16, size=(n, k))
    codes, scales = ref.store(t_codes, np.full((n, 3), 0x38, np.uint8), 128)          # every scale 1
    dense = ref.decode(codes, scales, 1.0, n, k, 128)
    w = handle(qnn, t, codes[None], scales[None], np.ones(1, np.float32), n, k, 128)
    x, x64 = real(t, rng, (rows, k), dtype)
    x[1, 299], x[2, 17], x[2, 18] = float("inf"), float("nan"), float("-inf")
    y = qnn.g4_matvec(x, w).cpu().double().numpy()
    mag = np.abs(x64) @ np.abs(dense).T
    for r in (0, 3):
        assert np.all(np.abs(y[r] - x64[r] @ dense.T) <= ref.bound(x64[r] @ dense.T, mag[r], k, dtype))
    assert np.array_equal(y[1], np.sign(dense[:, 299]) * np.inf)
    assert np.all(np.isnan(y[2]))


def test_matvec_largest_fp32_values(t, qnn):
    """fp32 rows near the ends of the range enter exactly: one nonzero product a sum, so the result has one rounding."""
    n, k = 16, 64
    rng = np.random.default_rng(7)
    codes, scales = ref.store(np.full((n, k), 8), np.full((n, 1), 0x18, np.uint8), 128)      # W = 1/16
    dense = ref.decode(codes, scales, 1.0, n, k, 128)
    w = handle(qnn, t, codes[None], scales[None], np.ones(1, np.float32), n, k, 128)
    x = np.zeros((6, k), np.float32)
    x[np.arange(6), rng.integers(0, k, 6)] = np.array([3.4028235e38, -3.4028235e38, 1.17549435e-30, 1.0000001, 16777215.0, -7.0e-20], np.float32)
    y = qnn.g4_matvec(t.from_numpy(x).to(DEV), w).cpu().double().numpy()
    want = x.astype(np.float64) @ dense.T
    assert np.all(np.abs(y - want) <= 2.0 ** -23 * np.abs(want))


# ------------------------------------------------------------------------------------------------ grouped by expert

COUNTS = [[1], [0, 1], [3, 0, 2], [40, 0, 1, 17], [130], [0, 0, 260, 0], [64, 129, 5, 0, 300]]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (130, 129, 128), (64, 520, 64), (257, 72, 32)])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_expert_gemm(t, qnn, dtype, n, k, group, counts):
    rng = np.random.default_rng(sum(counts) * 7919 + n + k)
    codes, scales, alpha, dense = ref.random_weights(rng, len(counts), n, k, group)
    x, x64 = real(t, rng, (sum(counts), k), dtype)
    y = qnn.g4_expert_gemm(x, handle(qnn, t, codes, scales, alpha, n, k, group), offsets_of(t, counts))
    want, mag = np.zeros((sum(counts), n)), np.zeros((sum(counts), n))

    def one(e, a, b):
        want[a:b], mag[a:b] = x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T
    grouped(counts, 0, one)
    check(y, want, mag, k, dtype)
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (130, 129, 128), (520, 64, 64), (72, 257, 32)])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_expert_backward_data(t, qnn, dtype, n, k, group, counts):
    rng = np.random.default_rng(sum(counts) * 104729 + n + k)
    codes, scales, alpha, dense = ref.random_weights(rng, len(counts), n, k, group)
    dy, dy64 = real(t, rng, (sum(counts), n), dtype)
    dx = qnn.g4_expert_gemm_backward_data(dy, handle(qnn, t, codes, scales, alpha, n, k, group), offsets_of(t, counts))
    want, mag = np.zeros((sum(counts), k)), np.zeros((sum(counts), k))

    def one(e, a, b):
        want[a:b], mag[a:b] = dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e])
    grouped(counts, 0, one)
    check(dx, want, mag, n, dtype)
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (130, 129), (64, 520), (257, 72)])
@pytest.mark.parametrize("counts", COUNTS + [[0, 0]], ids=str)
def test_expert_backward_weights(t, qnn, dtype, n, k, counts):
    rng = np.random.default_rng(sum(counts) * 15485863 + n + k)
    rows = sum(counts)
    dy, dy64 = real(t, rng, (rows, n), dtype)
    x, x64 = real(t, rng, (rows, k), dtype)
    gw = t.full((len(counts), n, k), float("nan"), device=DEV)
    qnn.expert_gemm_backward_weights(dy, x, offsets_of(t, counts), gw=gw)
    want, mag = np.zeros((len(counts), n, k)), np.zeros((len(counts), n, k))

    def one(e, a, b):
        want[e], mag[e] = dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b])
    grouped(counts, 0, one)
    # two split operands: six products of parts, the dropped ones below 2^-23 of a product
    check(gw, want, mag, 2 * max(counts) + 64, "fp32")
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k,counts", [(70, 90, [2500, 0, 3]), (64, 64, [1111]), (300, 700, [900, 800])], ids=str)
def test_long_weight_gradients(t, qnn, dtype, n, k, counts):
    """Many rows on small matrices: sums of many blocks of rows, and rows split over the GPU."""
    rng = np.random.default_rng(n + k)
    rows = sum(counts)
    dy, dy64 = real(t, rng, (rows, n), dtype)
    x, x64 = real(t, rng, (rows, k), dtype)
    offsets = offsets_of(t, counts)
    gw = qnn.expert_gemm_backward_weights(dy, x, offsets)
    want, mag = np.zeros((len(counts), n, k)), np.zeros((len(counts), n, k))

    def one(e, a, b):
        want[e], mag[e] = dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b])
    grouped(counts, 0, one)
    check(gw, want, mag, 2 * max(counts) + 64, "fp32")
    # in the mean the sums are far better than that bound: kept to nearest, they do not drift towards zero
    assert np.linalg.norm(gw.cpu().double().numpy() - want) <= 1e-6 * np.linalg.norm(want)
    assert t.equal(gw, qnn.expert_gemm_backward_weights(dy, x, offsets)) and qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k,counts", [(256, 4000, [40, 30]), (2050, 256, [40, 30]), (1408, 1920, [300, 0, 200, 17])], ids=str)
def test_long_contractions_and_many_tiles(t, qnn, dtype, n, k, counts):
    """Rings that go round many times, blocks that take many tiles, in both directions."""
    rng = np.random.default_rng(n * 3 + k)
    codes, scales, alpha, dense = ref.random_weights(rng, len(counts), n, k, 64)
    w = handle(qnn, t, codes, scales, alpha, n, k, 64)
    rows = sum(counts)
    x, x64 = real(t, rng, (rows, k), dtype)
    dy, dy64 = real(t, rng, (rows, n), dtype)
    offsets = offsets_of(t, counts)
    y, dx = qnn.g4_expert_gemm(x, w, offsets), qnn.g4_expert_gemm_backward_data(dy, w, offsets)

    def one(e, a, b):
        check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, dtype)
        check(dx[a:b], dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e]), n, dtype)
    grouped(counts, 0, one)
    assert qnn.tensor_path_status() == 0


def test_fp32_products_do_not_drift(t, qnn):
    """fp32 results of a long contraction stay at fp32 accuracy in the mean."""
    rng = np.random.default_rng(21)
    n, k, counts = 256, 4096, [200, 100]
    codes, scales, alpha, dense = ref.random_weights(rng, 2, n, k, 128)
    w = handle(qnn, t, codes, scales, alpha, n, k, 128)
    x, x64 = real(t, rng, (300, k), "fp32")
    y = qnn.g4_expert_gemm(x, w, offsets_of(t, counts)).cpu().double().numpy()
    want = np.concatenate([x64[:200] @ dense[0].T, x64[200:] @ dense[1].T])
    assert np.linalg.norm(y - want) <= 1e-6 * np.linalg.norm(want)
    few = qnn.g4_matvec(x[:3], qnn.G4Weights(w.codes[:1], w.scales[:1], w.alpha[:1], n, k, 128)).cpu().double().numpy()
    assert np.linalg.norm(few - want[:3]) <= 1e-6 * np.linalg.norm(want[:3])


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_rows_of_no_expert_are_left_alone(t, qnn, dtype):
    """Rows in front of the first and behind the last expert hold NaN and take no part; their results are not written."""
    rng = np.random.default_rng(11)
    n, k, counts, lead, rows = 140, 200, [9, 0, 70], 5, 100
    codes, scales, alpha, dense = ref.random_weights(rng, 3, n, k, 64)
    w = handle(qnn, t, codes, scales, alpha, n, k, 64)
    x, x64 = real(t, rng, (rows, k), dtype)
    dy, dy64 = real(t, rng, (rows, n), dtype)
    inside = np.zeros(rows, bool)
    inside[lead:lead + sum(counts)] = True
    outside = t.from_numpy(~inside).to(DEV)
    x[outside], dy[outside] = float("nan"), float("inf")
    offsets = offsets_of(t, counts, lead)
    y = t.full((rows, n), 77.0, dtype=x.dtype, device=DEV)
    dx = t.full((rows, k), 77.0, dtype=x.dtype, device=DEV)
    qnn.g4_expert_gemm(x, w, offsets, out=y)
    qnn.g4_expert_gemm_backward_data(dy, w, offsets, out=dx)
    gw = qnn.expert_gemm_backward_weights(dy, x, offsets)
    assert bool((y[outside] == 77.0).all()) and bool((dx[outside] == 77.0).all())
    ww = np.zeros((3, n, k))
    wm = np.zeros((3, n, k))

    def one(e, a, b):
        check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, dtype)
        check(dx[a:b], dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e]), n, dtype)
        ww[e], wm[e] = dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b])
    grouped(counts, lead, one)
    check(gw, ww, wm, 2 * max(counts) + 64, "fp32")


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_nan_of_one_expert_stays_there(t, qnn, dtype):
    """A block of rows that the hardware fetches whole crosses into the next expert's rows; its values must not count."""
    rng = np.random.default_rng(12)
    n, k, counts = 136, 144, [33, 50, 20]
    codes, scales, alpha, dense = ref.random_weights(rng, 3, n, k, 128)
    w = handle(qnn, t, codes, scales, alpha, n, k, 128)
    x, x64 = real(t, rng, (103, k), dtype)
    dy, dy64 = real(t, rng, (103, n), dtype)
    x[33:83], dy[33:83] = float("nan"), float("nan")
    offsets = offsets_of(t, counts)
    y, dx, gw = qnn.g4_expert_gemm(x, w, offsets), qnn.g4_expert_gemm_backward_data(dy, w, offsets), qnn.expert_gemm_backward_weights(dy, x, offsets)
    assert bool(y[33:83].isnan().all()) and bool(dx[33:83].isnan().all()) and bool(gw[1].isnan().all())
    for e, a, b in ((0, 0, 33), (2, 83, 103)):
        check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, dtype)
        check(dx[a:b], dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e]), n, dtype)
        check(gw[e], dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b]), 2 * (b - a) + 64, "fp32")


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_expert_strides_and_alignment(t, qnn, dtype):
    rng = np.random.default_rng(13)
    n, k, counts = 90, 170, [20, 45]
    rows = sum(counts)
    codes, scales, alpha, dense = ref.random_weights(rng, 2, n, k, 32)
    w = handle(qnn, t, codes, scales, alpha, n, k, 32)
    xb, xb64 = real(t, rng, (rows, 200), dtype)
    db, db64 = real(t, rng, (rows, 120), dtype)
    offsets = offsets_of(t, counts)
    for at in (0, 1, 8):
        x, x64, dy, dy64 = xb[:, at:at + k], xb64[:, at:at + k], db[:, at:at + n], db64[:, at:at + n]
        y = qnn.g4_expert_gemm(x, w, offsets, out=t.empty((rows, n + 5), dtype=x.dtype, device=DEV)[:, 1:1 + n])
        dx = qnn.g4_expert_gemm_backward_data(dy, w, offsets, out=t.empty((rows, k + 5), dtype=x.dtype, device=DEV)[:, 3:3 + k])
        gw = qnn.expert_gemm_backward_weights(dy, x, offsets)
        for e, a, b in ((0, 0, 20), (1, 20, 65)):
            check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, dtype)
            check(dx[a:b], dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e]), n, dtype)
            check(gw[e], dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b]), 2 * (b - a) + 64, "fp32")


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_zero_rows(t, qnn, dtype):
    rng = np.random.default_rng(14)
    codes, scales, alpha, _ = ref.random_weights(rng, 2, 40, 50, 64)
    w = handle(qnn, t, codes, scales, alpha, 40, 50, 64)
    x = t.empty((0, 50), dtype=ref.torch_type(dtype), device=DEV)
    dy = t.empty((0, 40), dtype=ref.torch_type(dtype), device=DEV)
    offsets = offsets_of(t, [0, 0])
    assert qnn.g4_expert_gemm(x, w, offsets).shape == (0, 40)
    assert qnn.g4_expert_gemm_backward_data(dy, w, offsets).shape == (0, 50)
    gw = t.full((2, 40, 50), float("nan"), device=DEV)
    assert bool((qnn.expert_gemm_backward_weights(dy, x, offsets, gw=gw) == 0).all())


@pytest.mark.parametrize("counts", [[5, 9], [600, 200]], ids=str)
def test_gradients_against_differences(t, qnn, counts):
    """y is linear in x and in the decoded weights, so a central difference has no truncation error: <dy, f(x + d) - f(x - d)> / 2
    = <dx, d>, and <dy, x D^T> = <gw, D>.  fp32; bound: every inner product's sums, as in g4_reference.bound."""
    rng = np.random.default_rng(15)
    n, k, group = 150, 220, 64
    rows = sum(counts)
    codes, scales, alpha, dense = ref.random_weights(rng, 2, n, k, group)
    w = handle(qnn, t, codes, scales, alpha, n, k, group)
    x, x64 = real(t, rng, (rows, k), "fp32")
    d, d64 = real(t, rng, (rows, k), "fp32")
    dy, dy64 = real(t, rng, (rows, n), "fp32")
    offsets = offsets_of(t, counts)
    up, down = qnn.g4_expert_gemm(x + d, w, offsets), qnn.g4_expert_gemm(x - d, w, offsets)
    dx = qnn.g4_expert_gemm_backward_data(dy, w, offsets)
    lhs = float((dy.double() * (up.double() - down.double())).sum() / 2)
    rhs = float((dx.double() * d.double()).sum())
    mag = 0.0
    for e, (a, b) in enumerate(((0, counts[0]), (counts[0], rows))):
        m = (np.abs(x64[a:b]) + np.abs(d64[a:b])) @ np.abs(dense[e]).T
        mag += float((np.abs(dy64[a:b]) * m).sum())
    assert abs(lhs - rhs) <= (3 * max(n, k) + 80) * 2.0 ** -23 * 2 * mag
    # weights: move one expert's weights by another expert's (a handle with the same rows, other codes)
    swapped = handle(qnn, t, codes[::-1].copy(), scales[::-1].copy(), alpha[::-1].copy(), n, k, group)
    gw = qnn.expert_gemm_backward_weights(dy, x, offsets).cpu().double().numpy()
    y0, y1 = qnn.g4_expert_gemm(x, w, offsets).double(), qnn.g4_expert_gemm(x, swapped, offsets).double()
    lhs = float((dy.double() * (y1 - y0)).sum())
    rhs = sum(float((gw[e] * (dense[1 - e] - dense[e])).sum()) for e in range(2))
    mag = 0.0
    for e, (a, b) in enumerate(((0, counts[0]), (counts[0], rows))):
        mag += float((np.abs(dy64[a:b]) * (np.abs(x64[a:b]) @ (np.abs(dense[0]) + np.abs(dense[1])).T)).sum())
    assert abs(lhs - rhs) <= (3 * max(k, rows) + 80) * 2.0 ** -23 * 2 * mag


def test_same_bits_every_call_and_every_stream(t, qnn):
    """No result depends on timing: sums run in a fixed order.  A side stream gives the same bits."""
    rng = np.random.default_rng(16)
    n, k, counts = 300, 400, [70, 1, 200]
    codes, scales, alpha, _ = ref.random_weights(rng, 3, n, k, 64)
    w = handle(qnn, t, codes, scales, alpha, n, k, 64)
    x, _ = real(t, rng, (271, k), "fp32")
    dy, _ = real(t, rng, (271, n), "fp32")
    offsets = offsets_of(t, counts)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    for f in (lambda s: qnn.g4_expert_gemm(x, w, offsets, stream=s), lambda s: qnn.g4_expert_gemm_backward_data(dy, w, offsets, stream=s),
              lambda s: qnn.expert_gemm_backward_weights(dy, x, offsets, stream=s),
              lambda s: qnn.g4_matvec(x[:7], qnn.G4Weights(w.codes[:1], w.scales[:1], w.alpha[:1], n, k, 64), stream=s)):
        a = f(None)
        others = [f(side) for _ in range(3)] + [f(None)]
        t.cuda.synchronize()
        assert all(t.equal(a, o) for o in others)


def test_captured_call_follows_new_offsets(t, qnn):
    """The split of the rows is read on the device: a captured graph replays with another one."""
    rng = np.random.default_rng(17)
    n, k, rows = 136, 136, 90
    codes, scales, alpha, dense = ref.random_weights(rng, 3, n, k, 128)
    w = handle(qnn, t, codes, scales, alpha, n, k, 128)
    x, x64 = real(t, rng, (rows, k), "bf16")
    dy, dy64 = real(t, rng, (rows, n), "bf16")
    offsets = offsets_of(t, [30, 30, 30])
    y, dx, gw = t.empty((rows, n), dtype=x.dtype, device=DEV), t.empty((rows, k), dtype=x.dtype, device=DEV), t.empty((3, n, k), device=DEV)

    def step():
        qnn.g4_expert_gemm(x, w, offsets, out=y)
        qnn.g4_expert_gemm_backward_data(dy, w, offsets, out=dx)
        qnn.expert_gemm_backward_weights(dy, x, offsets, gw=gw)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        step()
    side.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        step()
    for counts in ([90, 0, 0], [1, 0, 89], [20, 41, 29]):
        offsets.copy_(offsets_of(t, counts))
        graph.replay()
        t.cuda.synchronize()

        def one(e, a, b):
            check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, "bf16")
            check(dx[a:b], dy64[a:b] @ dense[e], np.abs(dy64[a:b]) @ np.abs(dense[e]), n, "bf16")
            check(gw[e], dy64[a:b].T @ x64[a:b], np.abs(dy64[a:b]).T @ np.abs(x64[a:b]), 2 * (b - a) + 64, "fp32")
        grouped(counts, 0, one)


def test_offsets_out_of_range_are_clamped(t, qnn):
    """Offsets that leave 0 .. rows or decrease touch no memory outside the operands."""
    rng = np.random.default_rng(18)
    n, k, rows = 130, 130, 40
    codes, scales, alpha, dense = ref.random_weights(rng, 3, n, k, 128)
    w = handle(qnn, t, codes, scales, alpha, n, k, 128)
    x, x64 = real(t, rng, (rows, k), "bf16")
    dy, _ = real(t, rng, (rows, n), "bf16")
    for raw in ([-5, 10, 1 << 30, 1 << 30], [0, 40, 10, 40], [50, 60, 70, 80]):
        offsets = t.tensor(raw, dtype=t.int32, device=DEV)
        y = t.zeros((rows + 2, n), dtype=x.dtype, device=DEV)
        qnn.g4_expert_gemm(x, w, offsets, out=y[1:-1])
        qnn.g4_expert_gemm_backward_data(dy, w, offsets)
        qnn.expert_gemm_backward_weights(dy, x, offsets)
        t.cuda.synchronize()
        assert bool((y[0] == 0).all()) and bool((y[-1] == 0).all())
        if raw[0] == -5:
            check(y[1:11], x64[:10] @ dense[0].T, np.abs(x64[:10]) @ np.abs(dense[0]).T, k, "bf16")
    assert qnn.tensor_path_status() == 0


def test_many_experts(t, qnn):
    """More experts than a warp has lanes, most of them without rows."""
    rng = np.random.default_rng(19)
    n, k, experts = 70, 90, 100
    codes, scales, alpha, dense = ref.random_weights(rng, experts, n, k, 64)
    counts = np.zeros(experts, int)
    counts[[0, 31, 32, 33, 64, 99]] = [1, 2, 3, 140, 5, 6]
    x, x64 = real(t, rng, (157, k), "fp16")
    w = handle(qnn, t, codes, scales, alpha, n, k, 64)
    y = qnn.g4_expert_gemm(x, w, offsets_of(t, counts))
    some = qnn.g4_expert_gemm(x[:3], w, offsets_of(t, np.minimum(counts, [1] + 30 * [0] + [2] + 68 * [0])))
    grouped(counts, 0, lambda e, a, b: check(y[a:b], x64[a:b] @ dense[e].T, np.abs(x64[a:b]) @ np.abs(dense[e]).T, k, "fp16"))
    check(some[1:3], x64[1:3] @ dense[31].T, np.abs(x64[1:3]) @ np.abs(dense[31]).T, k, "fp16")


def test_experts_layer_runs_and_learns(t, qnn):
    """The layer of run_case: forward equals the same layer on decoded weights, training brings the loss down."""
    from paper_2106_09886_b200.run_case import ExpertsLayer
    layer = ExpertsLayer(192, 320, 6, 2, 200, group=64, dtype=t.float32, seed=3)
    g = t.Generator(device=DEV).manual_seed(4)
    x = t.randn((75, 192), device=DEV, generator=g)

    def dense(q):
        c, s = q.codes.cpu().numpy(), q.scales.cpu().numpy()
        return np.stack([ref.decode(c[e], s[e], q.alpha[e].item(), q.n, q.k, q.group) for e in range(c.shape[0])])
    token, gate, offsets = layer.plan(x)
    assert sorted(token.tolist()) == sorted(2 * list(range(75))) and offsets[-1].item() == 150
    w1, w2, x64 = dense(layer.q1), dense(layer.q2), x.cpu().double().numpy()
    want, bounds = np.zeros((75, 192)), offsets.tolist()
    for e in range(6):
        for r in range(bounds[e], bounds[e + 1]):
            h = w1[e] @ x64[token[r].item()]
            want[token[r].item()] += gate[r].item() * (w2[e] @ (h / (1 + np.exp(-h))))
    got = layer.forward(x)[0].cpu().double().numpy()
    assert np.linalg.norm(got - want) <= 1e-5 * np.linalg.norm(want)
    logits = layer.logits(x[:1])
    assert logits.shape == (1, 200) and bool(logits.isfinite().all())
    target = t.randn((75, 192), device=DEV, generator=g)
    losses = [layer.train_step(x, target, 0.5)[0] for _ in range(12)]
    assert losses[-1] < 0.9 * losses[0] and qnn.tensor_path_status() == 0

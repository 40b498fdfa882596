"""Rows with values near both ends of their type's range, times weights as the packer makes them (scale 448 in the largest group,
alpha = max|w| / 6720): a result that its type holds must not overflow, or lose its digits, on the way."""
import numpy as np
import pytest

import g4_reference as ref

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


def packed(qnn, t, rng, n, k, size):
    """Weights around `size` from the packer, and what they decode to in 64 bits."""
    w = qnn.g4_pack_weights(t.from_numpy((rng.standard_normal((n, k)) * size).astype(np.float32)).to(DEV), 64)
    dense = ref.decode(w.codes[0].cpu().numpy(), w.scales[0].cpu().numpy(), w.alpha[0].item(), n, k, 64)
    return w, dense


def few_values(t, rng, rows, width, size, dtype):
    """Two values of about `size` in each row and zeros elsewhere: sums are no larger than their terms' magnitudes."""
    v = np.zeros((rows, width), np.float32)
    for r in range(rows):
        at = rng.choice(width, 2, replace=False)
        v[r, at] = rng.choice([-1.0, 1.0], 2) * rng.uniform(0.5, 1.0, 2) * size
    v = t.from_numpy(v).to(ref.torch_type(dtype))
    return v.to(DEV), v.double().numpy()


def check(got, exact, magnitude, dtype):
    """Two terms: three parts each at most, so six additions, and one rounding to the type."""
    got = got.to("cpu").double().numpy()
    u, tiny = ref.ROUND[dtype]
    assert np.all(np.abs(got - exact) <= u * np.abs(exact) + 16 * 2.0 ** -23 * magnitude + tiny), np.max(np.abs(got - exact) / magnitude.max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [1, 3, 100])
@pytest.mark.parametrize("size,weight", [(1e36, 0.1), (1e38, 0.05), (1e37, 0.01), (1e-25, 0.05), (1.0, 1e-30), (1e-4, 1e33)])
def test_products_near_the_ends_of_the_range(t, qnn, dtype, rows, size, weight):
    rng = np.random.default_rng(rows + int(100 * abs(np.log10(size))))
    n, k = 130, 264
    w, dense = packed(qnn, t, rng, n, k, weight)
    offsets = t.tensor([0, rows], dtype=t.int32, device=DEV)
    x, x64 = few_values(t, rng, rows, k, size, dtype)
    dy, dy64 = few_values(t, rng, rows, n, size, dtype)
    want, mag = x64 @ dense.T, np.abs(x64) @ np.abs(dense).T
    assert mag.max() < 3e38
    check(qnn.g4_matvec(x, w), want, mag, dtype)
    check(qnn.g4_expert_gemm(x, w, offsets), want, mag, dtype)
    check(qnn.g4_expert_gemm_backward_data(dy, w, offsets), dy64 @ dense, np.abs(dy64) @ np.abs(dense), dtype)
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("rows", [3, 100])
def test_split_sums_near_the_end_of_the_range(t, qnn, rows):
    """A long contraction, which is split: the parts are results in themselves."""
    rng = np.random.default_rng(rows)
    n, k = 64, 4096
    w, dense = packed(qnn, t, rng, n, k, 0.05)
    for dtype in ("fp32", "bf16"):
        x, x64 = few_values(t, rng, rows, k, 1e38, dtype)
        check(qnn.g4_matvec(x, w), x64 @ dense.T, np.abs(x64) @ np.abs(dense).T, dtype)


@pytest.mark.parametrize("rows", [2, 100])
def test_smallest_values_that_enter_exactly(t, qnn, rows):
    """fp32 rows from 2^-79 up have all their 24 bits in the products, at the smallest scale too: one nonzero product a sum, three
    parts whose sums are exact, so the result has one rounding."""
    rng = np.random.default_rng(rows)
    n, k = 136, 200
    codes, scales = ref.store(rng.integers(7, 9, (n, k)), np.full((n, 2), 0x01, np.uint8), 128)         # W = +-2^-9
    dense = ref.decode(codes, scales, 1.0, n, k, 128)
    w = qnn.G4Weights(t.from_numpy(codes[None]).to(DEV), t.from_numpy(scales[None]).to(DEV), t.ones(1, device=DEV), n, k, 128)
    offsets = t.tensor([0, rows], dtype=t.int32, device=DEV)

    def ones(width):
        v = np.zeros((rows, width), np.float32)
        v[np.arange(rows), rng.integers(0, width, rows)] = ((2 ** 23 + rng.integers(0, 2 ** 23, rows)) * 2.0 ** -23 * 2.0 ** -79).astype(np.float32)
        return t.from_numpy(v).to(DEV), v.astype(np.float64)
    (x, x64), (dy, dy64) = ones(k), ones(n)
    for got, want in ((qnn.g4_matvec(x, w), x64 @ dense.T), (qnn.g4_expert_gemm(x, w, offsets), x64 @ dense.T),
                      (qnn.g4_expert_gemm_backward_data(dy, w, offsets), dy64 @ dense)):
        assert np.all(np.abs(got.cpu().double().numpy() - want) <= 2.0 ** -23 * np.abs(want))


@pytest.mark.parametrize("n,k", [(40, 48), (300, 264)])
def test_products_of_parts_that_are_left_out(t, qnn, n, k):
    """One row, so that every element of an fp32 weight gradient is one product: the parts left out are below 2^-21 of it, and the
    five additions of the six that are taken, which may cut, each below 2^-23.  A product too few of the first two parts would
    be 2^-16 off."""
    rng = np.random.default_rng(n)
    dy, x = rng.standard_normal((1, n)).astype(np.float32), rng.standard_normal((1, k)).astype(np.float32)
    gw = qnn.expert_gemm_backward_weights(t.from_numpy(dy).to(DEV), t.from_numpy(x).to(DEV), t.tensor([0, 1], dtype=t.int32, device=DEV))
    want = dy.astype(np.float64).T @ x.astype(np.float64)
    assert np.all(np.abs(gw[0].cpu().double().numpy() - want) <= (4 + 6) * 2.0 ** -23 * np.abs(want))


@pytest.mark.parametrize("counts", [[1], [3, 0, 2], [40, 0, 1, 17], [130], [64, 129, 5, 0, 300]], ids=str)
@pytest.mark.parametrize("n,k", [(130, 129), (257, 72)])
def test_fp32_weight_gradients_in_the_mean(t, qnn, counts, n, k):
    """In the 2-norm an fp32 weight gradient is within 1e-6 at every number of rows, not for long ones alone."""
    rng = np.random.default_rng(sum(counts) + n)
    rows = sum(counts)
    dy, x = rng.standard_normal((rows, n)).astype(np.float32), rng.standard_normal((rows, k)).astype(np.float32)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    gw = qnn.expert_gemm_backward_weights(t.from_numpy(dy).to(DEV), t.from_numpy(x).to(DEV), t.tensor(offsets, dtype=t.int32, device=DEV))
    want = np.stack([dy[a:b].astype(np.float64).T @ x[a:b].astype(np.float64) for a, b in zip(offsets, offsets[1:])])
    assert np.linalg.norm(gw.cpu().double().numpy() - want) <= 1e-6 * np.linalg.norm(want)

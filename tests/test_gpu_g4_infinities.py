"""Infinities and NaN among the real operands of the calls on 4-bit weights: a result holds what the formula gives in IEEE
arithmetic - an infinity times a finite number other than zero is an infinity, times zero a NaN - whatever parts a kernel
splits its operands into."""
import numpy as np
import pytest

import g4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def real(t, rng, shape, dtype, kind):
    """Values that fill one bf16 part ("short"), or as many bits as the type has ("full")."""
    v = rng.standard_normal(shape).astype(np.float32)
    v = t.from_numpy(v)
    if kind == "short":
        v = v.bfloat16().float()
    v = v.to(ref.torch_type(dtype))
    return v.to(DEV)


def same_specials(got, want):
    """Infinities with their signs and NaN where the formula has them, finite values where it has those."""
    got = got.to("cpu").double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(want), want, 0))


def plain(a, b):
    """a [m][r] times b [r][n] in 64 bits, term by term (a library product may skip zeros)."""
    with np.errstate(invalid="ignore"):
        return (a[:, :, None] * b[None, :, :]).sum(axis=1)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("dy_kind,x_kind", [("short", "short"), ("full", "short"), ("short", "full"), ("full", "full")])
@pytest.mark.parametrize("rows", [1, 70, 600])
def test_weight_gradient(t, qnn, dtype, dy_kind, x_kind, rows):
    rng = np.random.default_rng(rows)
    n, k = 40, 48
    dy, x = real(t, rng, (rows, n), dtype, dy_kind), real(t, rng, (rows, k), dtype, x_kind)
    at = rng.integers(0, rows, 6)
    x[at[0], 3], x[at[1], 5], x[at[2], 7] = INF, -INF, NAN
    dy[at[3], 2], dy[at[4], 4], dy[at[5], 6] = INF, -INF, NAN
    dy[at[0], 8] = 0.0                                                     # infinity times zero
    dy[at[0], 9], x[at[4], 9] = INF, -INF                                  # infinity times infinity
    offsets = t.tensor([0, rows], dtype=t.int32, device=DEV)
    gw = qnn.expert_gemm_backward_weights(dy, x, offsets)
    same_specials(gw[0], plain(dy.cpu().double().numpy().T, x.cpu().double().numpy()))
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("x_kind", ["short", "full"])
@pytest.mark.parametrize("rows", [1, 4, 90])
def test_products(t, qnn, dtype, x_kind, rows):
    """Few rows and tensor memory, forward and data gradient; some groups of weights are zeros."""
    rng = np.random.default_rng(100 + rows)
    n, k = 72, 200
    codes, scales, alpha, dense = ref.random_weights(rng, 1, n, k, 64)
    w = qnn.G4Weights(t.from_numpy(codes).to(DEV), t.from_numpy(scales).to(DEV), t.from_numpy(alpha).to(DEV), n, k, 64)
    offsets = t.tensor([0, rows], dtype=t.int32, device=DEV)
    x, dy = real(t, rng, (rows, k), dtype, x_kind), real(t, rng, (rows, n), dtype, x_kind)
    for v in (x, dy):
        v[rng.integers(0, rows), 3], v[rng.integers(0, rows), 5], v[rng.integers(0, rows), v.shape[1] - 1] = INF, -INF, INF
    v64 = x.cpu().double().numpy()
    want = plain(v64, dense[0].T)
    assert (dense[0] == 0).any()
    same_specials(qnn.g4_matvec(x, w), want)
    same_specials(qnn.g4_expert_gemm(x, w, offsets), want)
    same_specials(qnn.g4_expert_gemm_backward_data(dy, w, offsets), plain(dy.cpu().double().numpy(), dense[0]))
    assert qnn.tensor_path_status() == 0


def test_parts_of_an_infinity_beside_the_largest_values(t, qnn):
    """An infinity among the largest finite fp32 values, and those alone: no part of a finite value turns into an infinity."""
    n, k, rows = 32, 32, 64
    x = t.full((rows, k), 1.0, device=DEV)
    x[:, 0], x[:, 1] = 0.0, 0.0
    x[5, 0], x[5, 1] = float(np.float32(3.4028235e38)), INF
    dy = t.zeros((rows, n), device=DEV)
    dy[5] = 1.0
    gw = qnn.expert_gemm_backward_weights(dy, x, t.tensor([0, rows], dtype=t.int32, device=DEV))[0].cpu().double().numpy()
    with np.errstate(invalid="ignore"):
        want = dy.cpu().double().numpy().T @ np.where(np.isinf(x.cpu().double().numpy()), 0, x.cpu().double().numpy())
    assert np.all(np.abs(gw[:, 0] - want[:, 0]) <= 2.0 ** -23 * np.abs(want[:, 0]))          # one product: three parts, added
    assert np.array_equal(gw[:, 2:], want[:, 2:])
    assert np.all(gw[:, 1] == INF)

"""Calls on 4-bit weights that follow one another with nothing between them, each reading what the one before has just written:
their kernels start while the ones ahead still run, so what they read has to come from after those have ended.  Every result
must have the same bits as when the device is waited for between the calls."""
import numpy as np
import pytest

import g4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUNDS = 12


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


def handle(qnn, t, rng, experts, n, k, group):
    codes, scales, alpha, _ = ref.random_weights(rng, experts, n, k, group)
    return qnn.G4Weights(t.from_numpy(codes).to(DEV), t.from_numpy(scales).to(DEV), t.from_numpy(alpha * 100).to(DEV), n, k, group)


def both_ways(t, step, outputs):
    """step(i, sync) for every round: once with a wait for the device after each call, then all rounds queued at once."""
    for i in range(ROUNDS):
        step(i, t.cuda.synchronize)
    want = [o.clone() for o in outputs]
    for o in outputs:
        o.fill_(float("nan"))
    t.cuda.synchronize()
    for i in range(ROUNDS):
        step(i, lambda: None)
    t.cuda.synchronize()
    for i, (a, b) in enumerate(zip(outputs, want)):
        assert t.equal(a, b), f"output {i}"                      # (a NaN is not equal to itself: everything has been written)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,pad", [(8, 0), (8, 1), (300, 0), (300, 1), (1500, 0), (1500, 3)])
def test_product_into_product(t, qnn, dtype, rows, pad):
    """y of one grouped product is the next one's x: where it lies (aligned), or rewritten first (rows that are not)."""
    rng = np.random.default_rng(rows + pad)
    kind = ref.torch_type(dtype)
    up, down = handle(qnn, t, rng, 3, 392, 264, 64), handle(qnn, t, rng, 3, 264, 392, 128)
    offsets = t.tensor([0, rows // 3, rows // 2, rows], dtype=t.int32, device=DEV)
    xs = [t.from_numpy(rng.standard_normal((rows, 264)).astype(np.float32)).to(DEV).to(kind) for _ in range(ROUNDS)]
    y = t.zeros((rows, 392 + pad), dtype=kind, device=DEV)[:, :392]              # one buffer, written anew in each round
    zs = [t.zeros((rows, 264), dtype=kind, device=DEV) for _ in range(ROUNDS)]
    dxs = [t.zeros((rows, 264), dtype=kind, device=DEV) for _ in range(ROUNDS)]

    def step(i, sync):
        qnn.g4_expert_gemm(xs[i], up, offsets, out=y)
        sync()
        qnn.g4_expert_gemm(y, down, offsets, out=zs[i])
        sync()
        qnn.g4_expert_gemm_backward_data(y, up, offsets, out=dxs[i])
        sync()
    both_ways(t, step, zs + dxs)
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,pad", [(1, 0), (4, 1), (9, 0), (40, 1)])
def test_matvec_into_matvec(t, qnn, dtype, rows, pad):
    rng = np.random.default_rng(rows * 10 + pad)
    kind = ref.torch_type(dtype)
    up, down = handle(qnn, t, rng, 1, 1000, 520, 32), handle(qnn, t, rng, 1, 520, 1000, 64)
    xs = [t.from_numpy(rng.standard_normal((rows, 520)).astype(np.float32)).to(DEV).to(kind) for _ in range(ROUNDS)]
    y = t.zeros((rows, 1000 + pad), dtype=kind, device=DEV)[:, :1000]
    zs = [t.zeros((rows, 520), dtype=kind, device=DEV) for _ in range(ROUNDS)]

    def step(i, sync):
        qnn.g4_matvec(xs[i], up, out=y)
        sync()
        qnn.g4_matvec(y, down, out=zs[i])
        sync()
    both_ways(t, step, zs)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,k,rows", [(64, 72, 1500), (264, 392, 900)])
def test_weight_gradients_back_to_back(t, qnn, dtype, n, k, rows):
    """Rows split over the GPU: the parts of all calls share one workspace, the sum of one call is followed by the parts of the next."""
    rng = np.random.default_rng(n + rows)
    kind = ref.torch_type(dtype)
    w = handle(qnn, t, rng, 1, n, k, 64)
    offsets = t.tensor([0, rows], dtype=t.int32, device=DEV)
    dys = [t.from_numpy(rng.standard_normal((rows, n)).astype(np.float32)).to(DEV).to(kind) for _ in range(ROUNDS)]
    dx = t.zeros((rows, k), dtype=kind, device=DEV)
    need = qnn.lib.qnn_expert_backward_weights_workspace(dys[0].data_ptr(), dx.data_ptr(), qnn.REAL_TYPES[kind], rows, n, k, 1, n, k)
    assert need > 0
    workspace = t.zeros(need, dtype=t.uint8, device=DEV)
    gws = [t.zeros((1, n, k), device=DEV) for _ in range(ROUNDS)]

    def step(i, sync):
        qnn.g4_expert_gemm_backward_data(dys[i], w, offsets, out=dx)
        sync()
        qnn.expert_gemm_backward_weights(dys[i], dx, offsets, gw=gws[i], workspace=workspace)
        sync()
    both_ways(t, step, gws)
    assert qnn.tensor_path_status() == 0


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_experts_that_claim_the_same_rows_end_in_bounds(t, qnn, dtype):
    """Offsets that go back and forth between 0 and the number of rows, against the contract: the calls end, report nothing, and
    write inside their results only."""
    rng = np.random.default_rng(31)
    experts, n, k, rows = 40, 136, 72, 200
    w = handle(qnn, t, rng, experts, n, k, 64)
    kind = ref.torch_type(dtype)
    x = t.from_numpy(rng.standard_normal((rows, k)).astype(np.float32)).to(DEV).to(kind)
    dy = t.from_numpy(rng.standard_normal((rows, n)).astype(np.float32)).to(DEV).to(kind)
    offsets = t.tensor([0, rows] * 20 + [0], dtype=t.int32, device=DEV)
    y, dx = t.full((rows + 2, n), 5.0, dtype=kind, device=DEV), t.full((rows + 2, k), 5.0, dtype=kind, device=DEV)
    for many in (rows, 60):                                   # tiles for the tensor memory, and the form for few rows
        qnn.g4_expert_gemm(x[:many], w, offsets, out=y[1:many + 1])
        qnn.g4_expert_gemm_backward_data(dy[:many], w, offsets, out=dx[1:many + 1])
        t.cuda.synchronize()
        assert bool((y[[0, -1]] == 5.0).all()) and bool((dx[[0, -1]] == 5.0).all())
    assert qnn.tensor_path_status() == 0

"""Every tile of the grouped 4-bit products, its pairs of blocks among them, in both directions and for weight gradients: experts
of ragged sizes, rows that belong to nobody, one expert full of NaN, results that start and end inside 16 bytes, each against
64 bits (bounds: g4_reference.bound) and twice for its bits.  tests/test_g4_plans.py checks that the sizes take the tiles."""
import numpy as np
import pytest

import g4_reference as ref
import g4_shapes

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


def ragged(rng, rows, experts):
    """Offsets with rows of nobody at both ends (three and two, where there are enough), an expert of one row and one without."""
    lead, tail = (3, 2) if rows >= 20 else (0, 0)
    inner = rows - lead - tail
    if experts == 1:
        counts = [inner]
    elif experts == 2:
        counts = [1, inner - 1]
    else:
        counts = [0] * experts
        counts[1] = 1
        share = rng.uniform(0.4, 1.6, experts - 2)
        for e, c in zip(range(2, experts), rng.multinomial(inner - 1, share / share.sum())):
            counts[e] = int(c)
        counts[0], counts[2] = counts[2], 0
    return np.concatenate([[lead], lead + np.cumsum(counts)])


def check(got, exact, magnitude, length, dtype):
    got, exact, magnitude = (v.double().cpu().numpy() for v in (got, exact, magnitude))
    err, tol = np.abs(got - exact), ref.bound(exact, magnitude, length, dtype)
    assert np.all(err <= tol), f"worst {np.max(err / tol):.3g} of its bound"


def rows_of(t, rng, shape, dtype, gap):
    """Random rows whose stride is `gap` elements longer than they are."""
    v = t.from_numpy(rng.standard_normal((shape[0], shape[1] + gap)).astype(np.float32)).to(ref.torch_type(dtype)).to(DEV)
    return v[:, :shape[1]]


@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("product,dtype,rows,experts,n,k,tile,split", [s for s in g4_shapes.EVERY if s[0] != "weights"])
def test_products(t, qnn, product, dtype, rows, experts, n, k, tile, split, aligned):
    rng = np.random.default_rng(rows * 31 + n + k + tile)
    width, features = (k, n) if product == "experts" else (n, k)
    made = [ref.random_weights(rng, 1, n, k, (32, 64, 128)[e % 3] if experts == 1 else 64) for e in range(min(experts, 4))]
    which = [e % len(made) for e in range(experts)]
    group = 32 if experts == 1 else 64
    codes, scales, alpha = (np.concatenate([made[i][j] for i in which]) for j in range(3))
    dense = [t.from_numpy(m[3][0]).to(DEV) for m in made]
    w = qnn.G4Weights(t.from_numpy(codes).to(DEV), t.from_numpy(scales).to(DEV), t.from_numpy(alpha).to(DEV), n, k, group)
    bounds = ragged(rng, rows, experts)
    offsets = t.tensor(bounds, dtype=t.int32, device=DEV)
    gap = -width % 8 if aligned else 1 + -width % 2
    x = rows_of(t, rng, (rows, width), dtype, gap)
    sizes = np.diff(bounds)
    sick = int(np.argsort(sizes)[-2]) if experts > 1 else -1               # the second largest expert
    if sick >= 0:
        x[bounds[sick]:bounds[sick + 1]] = float("nan")
    x[:bounds[0]], x[bounds[-1]:] = float("inf"), float("nan")
    x64 = x.double()
    full = t.full((rows, features + 16), 7.0, dtype=x.dtype, device=DEV)
    out = full[:, 8:8 + features] if aligned and features % 8 == 0 else full[:, 3:3 + features]
    f = qnn.g4_expert_gemm if product == "experts" else qnn.g4_expert_gemm_backward_data
    f(x, w, offsets, out=out)
    assert qnn.tensor_path_status() == 0
    first = out.clone()
    for e in range(experts):
        a, b = bounds[e], bounds[e + 1]
        if a == b:
            continue
        if e == sick:
            assert bool(out[a:b].isnan().all())
            continue
        d = dense[which[e]]
        d = d.t() if product == "experts" else d
        check(out[a:b], x64[a:b] @ d, x64[a:b].abs() @ d.abs(), width, dtype)
    # nothing else is written
    keep = t.ones_like(full, dtype=t.bool)
    at = (full.data_ptr() - out.data_ptr()) // -full.element_size()
    keep[bounds[0]:bounds[-1], at:at + features] = False
    assert bool((full[keep] == 7.0).all())
    for _ in range(3):
        f(x, w, offsets, out=out)
        assert t.equal(out.nan_to_num(nan=9.0), first.nan_to_num(nan=9.0))


@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("product,dtype,rows,experts,n,k,tile,split", [s for s in g4_shapes.EVERY if s[0] == "weights"])
def test_weight_gradients(t, qnn, product, dtype, rows, experts, n, k, tile, split, aligned):
    rng = np.random.default_rng(rows * 37 + n + k)
    bounds = ragged(rng, rows, experts)
    offsets = t.tensor(bounds, dtype=t.int32, device=DEV)
    dy = rows_of(t, rng, (rows, n), dtype, -n % 8 if aligned else 1 + -n % 2)
    x = rows_of(t, rng, (rows, k), dtype, -k % 8 if aligned else 1 + -k % 2)
    sick = int(np.argsort(np.diff(bounds))[-2])
    dy[bounds[sick]:bounds[sick + 1]] = float("nan")
    for v in (dy, x):
        v[:bounds[0]], v[bounds[-1]:] = float("inf"), float("nan")
    whole = t.full((experts * n * k + 2,), 7.0, device=DEV)
    gw = whole[1:-1].view(experts, n, k)
    qnn.expert_gemm_backward_weights(dy, x, offsets, gw=gw)
    assert qnn.tensor_path_status() == 0
    first = gw.clone()
    for e in range(experts):
        a, b = bounds[e], bounds[e + 1]
        if e == sick:
            assert bool(gw[e].isnan().all())
            continue
        d64, x64 = dy[a:b].double(), x[a:b].double()
        # both operands split: their parts' additions, and what is left out (g4_reference.bound with twice the rows, and 2^-21)
        check(gw[e], d64.t() @ x64, d64.abs().t() @ x64.abs(), 2 * int(b - a) + 64, "fp32")
        want = d64.t() @ x64
        assert float((gw[e].double() - want).norm()) <= 1e-6 * float(want.norm())
    assert float(whole[0]) == 7.0 and float(whole[-1]) == 7.0
    for _ in range(3):
        qnn.expert_gemm_backward_weights(dy, x, offsets, gw=gw)
        assert t.equal(gw.nan_to_num(nan=9.0), first.nan_to_num(nan=9.0))

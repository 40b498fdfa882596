"""The gradient of routing for tokens that have no expert: padding whose logits and weights' gradients hold anything, and tokens whose
logits are not numbers."""
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


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("experts,top", [(8, 2), (40, 6), (160, 32), (1000, 5)])
def test_tokens_without_experts(t, qnn, dtype, score, renormalise, experts, top):
    rng = np.random.default_rng(experts + top)
    tokens = 30
    l = t.from_numpy(rng.standard_normal((tokens, experts)).astype(np.float32)).to(ref.torch_type(dtype)).to(DEV)
    inf, nan = float("inf"), float("nan")
    padding = t.zeros(tokens, dtype=t.bool, device=DEV)
    padding[3:12] = True
    l[3] = nan
    l[4, experts - 1] = nan
    l[5, 0] = inf
    l[6] = inf
    l[7] = -inf
    l[8, 1], l[8, 2] = inf, -inf
    l[9, 3], l[9, 4] = inf, nan
    l[10] = t.finfo(l.dtype).max
    l[13, 5] = nan                                                # not padding: weights NaN, no expert
    l[14] = -inf                                                  # nothing is left of it
    l[15, 1] = -inf                                               # one expert less
    none = padding.clone()
    none[13:15] = True
    routes = qnn.route(l, top, score, renormalise=renormalise, factor=1.5, mask=~padding)
    assert bool((routes.experts[none] == -1).all()) and bool((routes.experts[~none][:, 0] >= 0).all())
    dw = rng.standard_normal((tokens, top)).astype(np.float32)
    dw[3, 0], dw[4, 1], dw[13, 0] = nan, inf, nan
    got = qnn.route_backward(t.from_numpy(dw).to(DEV), l, routes.experts, score, renormalise, 1.5)
    assert bool((got[none] == 0).all())
    keep = ~none.cpu().numpy()
    l64, chosen = l.cpu().double().numpy()[keep], routes.experts.cpu().numpy()[keep]
    want, size = ref.route_backward(dw.astype(np.float64)[keep], l64, chosen, score, renormalise, 1.5)
    err = np.abs(got.cpu().double().numpy()[keep] - want)
    assert np.all(err <= ref.route_backward_bound(want, size, l64, dtype))

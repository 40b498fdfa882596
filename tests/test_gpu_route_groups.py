"""Groups of experts: those of 32 whose count is no power of two, sums of two keys that fp32 does not hold, and groups of which fewer than
two experts are left."""
import numpy as np
import pytest

import layer_reference as ref
from test_gpu_route import check, logits_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = np.float32(np.inf)
MOST = np.finfo(np.float32).max


@pytest.fixture(scope="module")
def t():
    import torch
    return torch


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("experts,groups,top_groups,top", [(96, 3, 2, 6), (160, 5, 2, 8), (192, 6, 1, 4), (288, 9, 4, 8), (480, 15, 15, 32), (736, 23, 5, 3), (992, 31, 30, 8)])
def test_groups_of_32(t, qnn, score, biased, group_score, experts, groups, top_groups, top):
    rng = np.random.default_rng(experts + groups + top)
    bias = (rng.standard_normal(experts) * 0.1).astype(np.float32) if biased else None
    for tokens in (3, 150):
        check(t, qnn, logits_of(t, rng, tokens, experts), top, bias=bias, score=score, groups=groups, top_groups=top_groups, group_score=group_score)


def chosen_by_two(logits, top, score, bias, groups, top_groups):
    """The definition in 64 bits: a group's worth is the sum of its two largest keys, -infinity where there are not two."""
    s = ref.scores(logits, score)
    out = np.full((len(logits), top), -1)
    for i, l in enumerate(logits):
        key = np.where(l == -np.inf, -np.inf, s[i] + bias)
        two = np.sort(key.reshape(groups, -1), axis=1)[:, -2:]
        with np.errstate(invalid="ignore"):
            worth = np.where(two[:, 0] == -np.inf, -np.inf, two.sum(1))
        kept = np.argsort(-worth, kind="stable")[:top_groups]
        key = np.where(np.isin(np.arange(len(l)) // (len(l) // groups), kept), key, -np.inf)
        pick = [e for e in np.argsort(-key, kind="stable")[:top] if key[e] > -np.inf]
        out[i, :len(pick)] = pick
    return out


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups", [(24, 4), (128, 4), (256, 8), (160, 5), (64, 16)])
def test_sums_at_the_ends_of_fp32(t, qnn, score, experts, groups):
    """Biases of the type's largest and lowest numbers and of infinities: sums of two overflow, infinities of both signs meet."""
    each = experts // groups
    rng = np.random.default_rng(experts)
    biases = []
    b = (rng.standard_normal(experts) * 0.1).astype(np.float32)
    for kind in range(7):
        c = b.copy()
        if kind == 0:                                                 # whole groups at the lowest number, the last of them excluded
            c[each:] = -MOST
            c[-each:] = -INF
        elif kind == 1:                                               # sums beyond fp32, the later group's larger
            c[:2] = MOST * np.float32(0.7)
            c[each:each + 2] = MOST * np.float32(0.9)
            c[2 * each:2 * each + 2] = MOST * np.float32(0.8)
        elif kind == 2:                                               # the same below
            c[:] = -MOST
            c[2 * each:3 * each] = -MOST * np.float32(0.8)
            c[each:2 * each] = -MOST * np.float32(0.7)
        elif kind == 3:                                               # +infinity beside nothing: not two experts
            c[:each] = -INF
            c[1] = INF
        elif kind == 4:                                               # one left in each group
            c[:] = -INF
            c[::each] = b[::each]
            c[each + 1] = -MOST
        elif kind == 5:                                               # +infinities, more of them in the last group
            c[0], c[each], c[-3:] = INF, INF, INF
        else:                                                         # one expert at the largest, others at the lowest
            c[:] = -MOST
            c[each], c[2 * each] = MOST, MOST
        biases.append(c)
    for c in biases:
        for top_groups, top in ((1, 2), (2, 4), (groups - 1, 6)):
            for tokens in (5, 140):
                l = logits_of(t, rng, tokens, experts)
                l[1, 2:4] = -float("inf")
                got = qnn.route(l, top, score, t.from_numpy(c).to(DEV), groups, top_groups, "top2")
                want = chosen_by_two(l.cpu().double().numpy(), top, score, c.astype(np.float64), groups, top_groups)
                assert np.array_equal(got.experts.cpu().numpy(), want)
                assert bool(got.weights.isfinite().all())

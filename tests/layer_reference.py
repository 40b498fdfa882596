"""Plain 64-bit forms (numpy) of routing, the root-mean-square norm and rows in 8 bits, written from the formulas in include/qnn.h,
and bounds for what the kernels may be off by."""
import numpy as np

U32 = 2.0 ** -24                                          # half a step of fp32, relative
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
SMALLEST_STEP = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}
TYPES = ["fp32", "bf16", "fp16"]


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def rounding(value, dtype):
    """What rounding `value` to a type may change."""
    return np.abs(value) * HALF_STEP[dtype] + SMALLEST_STEP[dtype] / 2


# ------------------------------------------------------------------------------------------------ rows in 8 bits

def quantize(x):
    """fp32 rows -> (codes, scales), operation for operation in fp32."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        m = np.max(np.abs(x), axis=1)                     # NaN if any is
        finite = m <= np.finfo(np.float32).max
        scale = np.where(finite, np.maximum((m / np.float32(127)).astype(np.float32), np.float32(2.0 ** -126)), np.float32(np.nan)).astype(np.float32)
        q = np.rint((x / scale[:, None]).astype(np.float32))
    codes = np.where(finite[:, None], np.clip(np.where(np.isnan(q), 0, q), -127, 127), 0).astype(np.int8)
    return codes, scale


def gemm(x, sx, w, sw, bias, dtype):
    """Operation for operation: the whole sum, rounded to fp32, times the token's scale, times the feature's, plus the bias."""
    import torch
    acc = x.astype(np.int64) @ w.astype(np.int64).T
    with np.errstate(all="ignore"):
        y = acc.astype(np.float32) * sx[:, None].astype(np.float32) * sw[None, :].astype(np.float32)
        if bias is not None:
            y = y + bias[None, :].astype(np.float32)
    return torch.from_numpy(y.astype(np.float32)).to(torch_type(dtype))


# ------------------------------------------------------------------------------------------------ norm

def norm(h, gain, eps):
    """64-bit (y, rstd) of rows h."""
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h * gain[None, :] * rstd[:, None], rstd


# A thread adds at most 64 squares in a row, warps and blocks 10 partial sums more; all are positive, so the sum is off by at most 74
# roundings, its square root by half of them, and quotient, sum with eps, root and inverse by one each.
RSTD_ROUNDINGS = 74 / 2 + 4
Y_ROUNDINGS = RSTD_ROUNDINGS + 2


def norm_backward(dy, h, gain, rstd, dh):
    u = h * rstd[:, None]
    a = dy * gain[None, :]
    dx = rstd[:, None] * (a - u * np.mean(a * u, axis=1, keepdims=True))
    return dx + (0 if dh is None else dh), (dy * u).sum(0)


def norm_backward_bounds(dy, h, gain, rstd, dh, dtype):
    """The mean adds at most 64 + 10 products of three factors, and is divided; then each element is rounded at every step.  A column of
    dgain adds `rows / 296` products or fewer, then 8 sums of warps or none, then up to 37 + 5 partial sums."""
    u, a = np.abs(h * rstd[:, None]), np.abs(dy * gain[None, :])
    mean = np.mean(a * u, axis=1, keepdims=True)
    dx, _ = norm_backward(dy, h, gain, rstd, dh)
    off = rstd[:, None] * (3 * a + u * mean * (74 + 3 + 1 + 4)) * U32 + (np.abs(dx) + (0 if dh is None else np.abs(dh))) * U32
    return off + rounding(np.abs(dx) + off, dtype), (np.abs(dy) * u).sum(0) * (h.shape[0] // 296 + 1 + 8 + 37 + 5 + 2) * U32


# ------------------------------------------------------------------------------------------------ routing

def scores(logits, kind):
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return 1.0 / (1.0 + np.exp(-logits))
        m = np.max(logits, axis=1, keepdims=True)
        e = np.exp(logits - np.where(np.isfinite(m), m, 0.0))
        s = e.sum(1, keepdims=True)
        return np.where(s > 0, e / np.where(s > 0, s, 1.0), 0.0)


def route(logits, top, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renormalise=True, factor=1.0, mask=None):
    """(experts, weights in 64 bits, order, place, offsets)."""
    tokens, experts = logits.shape
    s = scores(logits, score)
    chosen, weights = np.full((tokens, top), -1, dtype=np.int64), np.zeros((tokens, top))
    for t in range(tokens):
        if mask is not None and not mask[t]:
            continue
        if np.isnan(logits[t]).any() or (score == "softmax" and (logits[t] == np.inf).any()):
            weights[t] = np.nan
            continue
        key = logits[t] if bias is None else s[t] + bias
        key = np.where((logits[t] == -np.inf) | np.isnan(key), -np.inf, key)
        if groups > 1:
            side = key if bias is not None or group_score == "max" else np.where(key == -np.inf, -np.inf, s[t])
            side = np.sort(side.reshape(groups, -1), axis=1)[:, ::-1]
            worth = side[:, 0] if group_score == "max" else side[:, 0] + side[:, 1]
            kept = np.argsort(-worth, kind="stable")[:top_groups]
            key = np.where(np.isin(np.arange(experts) // (experts // groups), kept), key, -np.inf)
        pick = np.argsort(-key, kind="stable")[:top]
        pick = pick[key[pick] > -np.inf]
        chosen[t, :len(pick)] = pick
        w = s[t][pick]
        if renormalise and len(pick):
            # shares, with the largest score's power taken out
            l = logits[t][pick]
            if score == "softmax":
                w = np.exp(l - l.max())
            else:
                w = np.exp(np.minimum(l, 0) - min(l.max(), 0)) / (1 + np.exp(-np.abs(l)))
            w = w / w.sum()
        weights[t, :len(pick)] = factor * w
    flat = chosen.reshape(-1)
    counts = np.bincount(flat[flat >= 0], minlength=experts)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    order = np.full(flat.size, -1, dtype=np.int64)
    rows = np.argsort(np.where(flat < 0, experts, flat), kind="stable")[:offsets[-1]]
    order[:offsets[-1]] = rows
    place = np.full(flat.size, -1, dtype=np.int64)
    place[rows] = np.arange(offsets[-1])
    return chosen, weights, order, place.reshape(chosen.shape), offsets


def weight_bound(weights, logits, top, score, renormalise):
    """Relative roundings of a weight: expf within two steps (4 halves), a difference of logits rounded to fp32 ahead of it, sums of
    at most 42 positive numbers (32 in a lane, ten over lanes), two quotients, the factor."""
    spread = np.abs(np.where(np.isfinite(logits), logits, 0.0)).max() * (2 if score == "softmax" else 1)
    return np.abs(weights) * (2 * 4 + 2 * spread + 42 + 6) * U32 + 2.0 ** -140


def route_backward(dweights, logits, chosen, score="softmax", renormalise=True, factor=1.0):
    tokens, experts = logits.shape
    s = scores(logits, score)
    out, size = np.zeros((tokens, experts)), np.zeros((tokens, experts))
    for t in range(tokens):
        there = [(i, e) for i, e in enumerate(chosen[t]) if 0 <= e < experts]
        if there:
            i, e = (np.array(v) for v in zip(*there))
            dw, c = factor * dweights[t, i], s[t][e]
            if renormalise:
                l = logits[t][e]
                if score == "softmax":
                    u = np.exp(l - l.max())
                    share, left = u / u.sum(), np.ones(len(e))
                else:
                    u = np.exp(np.minimum(l, 0) - min(l.max(), 0)) / (1 + np.exp(-np.abs(l)))
                    share, left = u / u.sum(), np.exp(-np.maximum(l, 0)) / (1 + np.exp(-np.abs(l)))
                np.add.at(out[t], e, share * (dw - (dw * share).sum()) * left)
                np.add.at(size[t], e, share * (np.abs(dw) + (np.abs(dw) * share).sum()) * left)
                continue
            if score == "sigmoid":
                left = np.exp(-np.maximum(logits[t][e], 0)) / (1 + np.exp(-np.abs(logits[t][e])))
                np.add.at(out[t], e, dw * c * left)
                np.add.at(size[t], e, np.abs(dw) * c * left)
                continue
            np.add.at(out[t], e, dw * c)
            np.add.at(size[t], e, np.abs(dw) * c)
            out[t] -= s[t] * (dw * c).sum()
            size[t] += s[t] * (np.abs(dw) * c).sum()
    return out, size


def route_backward_bound(out, size, logits, dtype):
    """size: the magnitudes that were added; roundings as for the weights, taken twice (a score enters a product of two)."""
    spread = np.abs(np.where(np.isfinite(logits), logits, 0.0)).max() * 2
    off = size * 2 * (2 * 4 + 2 * spread + 42 + 8) * U32 + 2.0 ** -140
    return off + rounding(np.abs(out) + off, dtype)

"""Plain 64-bit forms of the group-scaled 4-bit weight calls, and the error bounds their kernels are held to."""
from __future__ import annotations

import numpy as np

TYPES = ("fp32", "bf16", "fp16")
# unit roundoff of each type and the largest error of a result below its normal range
ROUND = {"fp32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25)}


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def e4m3_values():
    """The 128 values of the 1-4-3 floats with sign 0 (entry 127 is NaN)."""
    v = np.empty(128)
    for b in range(128):
        e, m = b >> 3, b & 7
        v[b] = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
    v[127] = np.nan
    return v


def e4m3_round(s):
    """Nearest 1-4-3 float of fp32 values in [0, 448], ties to the even byte."""
    v = e4m3_values()[:127]
    hi = np.clip(np.searchsorted(v, s, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = np.asarray(s, np.float64) - v[lo], v[hi] - np.asarray(s, np.float64)
    pick_hi = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(pick_hi, hi, lo).astype(np.uint8)


def tiles(v):
    return (v + 127) // 128


def quantize(w, group):
    """fp32 [n][k] -> (t [n][k], scale bytes [n][groups over whole tiles], alpha): the binary32 steps of the header."""
    f = np.float32
    n, k = w.shape
    alpha = f(np.abs(np.nan_to_num(w, nan=0.0)).max()) / f(15 * 448)
    full = np.zeros((n, tiles(k) * 128), dtype=f)
    full[:, :k] = w
    parts = full.reshape(n, -1, group)
    m = np.abs(np.nan_to_num(parts, nan=0.0)).max(axis=2)
    with np.errstate(divide="ignore", invalid="ignore"):
        s = np.minimum(m / f(f(15) * alpha), f(448)) if alpha > 0 else np.zeros_like(m)
        byte = e4m3_round(s)
        step = (alpha * e4m3_values()[byte].astype(f)).astype(f)
        v = parts / step[:, :, None]
    c = np.clip(np.where(np.isnan(v), f(-16), v), f(-16), f(16)).astype(f)
    u = (c * f(0.5) + f(8)).astype(f)
    t = np.clip(np.where(c > 0, np.floor(u), np.ceil(u) - 1), 0, 15).astype(np.int64)
    t[step == 0] = 0
    return t.reshape(n, -1)[:, :k], byte, alpha


def store(t, byte, group):
    """Codes and scale bytes of one matrix -> the arrays (codes int32, scales uint8) that the header describes, word by word."""
    n, k = t.shape
    tn, tk = tiles(n), tiles(k)
    codes = np.zeros((tn, tk, 4, 128, 4), dtype=np.uint32)
    row, col = np.indices((n, k))
    inner = col % 128
    j = inner % 8
    word = t.astype(np.uint32) << (4 * (j // 2) + 16 * (j % 2)).astype(np.uint32)
    np.bitwise_or.at(codes, (row // 128, col // 128, inner // 8 % 4, row % 128, inner // 32), word)
    scales = np.zeros((tn, tk, 128 // group, 128), dtype=np.uint8)
    grow, g = np.indices(byte.shape)
    scales[grow // 128, g // (128 // group), g % (128 // group), grow % 128] = byte
    return codes.view(np.int32), scales


def decode(codes, scales, alpha, n, k, group):
    """Arrays of one matrix -> float64 [n][k]."""
    row, col = np.indices((n, k))
    inner = col % 128
    j = inner % 8
    word = codes.view(np.uint32)[row // 128, col // 128, inner // 8 % 4, row % 128, inner // 32]
    t = (word >> (4 * (j // 2) + 16 * (j % 2)).astype(np.uint32)) & 15
    s = e4m3_values()[scales[row // 128, col // 128, inner // group, row % 128]]
    return (2.0 * t - 15.0) * s * np.float64(alpha)


def random_weights(rng, experts, n, k, group):
    """Random codes and scales (every code, scales over five powers of two, some zero) in storage and as float64 [experts][n][k]."""
    codes, scales, dense = [], [], []
    alpha = (rng.uniform(0.5, 2.0, experts) * 1e-3).astype(np.float32)
    for e in range(experts):
        t = rng.integers(0, 16, size=(n, k))
        byte = rng.integers(0x28, 0x50, size=(n, tiles(k) * 128 // group)).astype(np.uint8)
        byte[rng.random(byte.shape) < 0.05] = 0
        byte[:, (k + group - 1) // group:] = 0
        c, s = store(t, byte, group)
        codes.append(c)
        scales.append(s)
        dense.append(decode(c, s, alpha[e], n, k, group))
    return np.stack(codes), np.stack(scales), alpha, np.stack(dense)


def bound(exact, magnitude, length, dtype):
    """|got - exact| allowed: one rounding to the result's type, and for each of the `length` additions of a sum (and the few
    of a split operand) at most 2^-23 of the sum of magnitudes, which covers additions that truncate."""
    u, tiny = ROUND[dtype]
    acc = (3 * length + 64) * 2.0 ** -23 * magnitude if dtype == "fp32" else (length + 64) * 2.0 ** -23 * magnitude
    return u * np.abs(exact) + acc * (1 + u) + tiny

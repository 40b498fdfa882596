"""Timed cases of the group-scaled 4-bit weight operators: matrix-vector products, products grouped by expert, and the
backward products of the latter.

A weight matrix [n][k] is stored as one 4-bit odd code per element, one 8-bit float (1-4-3, finite, not negative) per
`group` consecutive elements of a row, and one fp32 factor alpha per matrix:

    W[j][i] = alpha * scale[j][i // group] * (2 t[j][i] - 15),     t in 0 .. 15

in tiles of 128 rows x 128 columns (padding rows and columns have scale 0):

    codes   int32 [experts][tiles_n][tiles_k][4 (c)][128 (row)][4 (w)]; the word holds the eight elements
            128*tile + 32*w + 8*c + j, j = 0 .. 7, element j = 2p + h at bits 4p + 16h
    scales  uint8 [experts][tiles_n][tiles_k][128 / group][128 (row)]
    alpha   fp32  [experts]

Rows of x (and dy) are sorted by expert: expert e has rows offsets[e] .. offsets[e+1].

    matvec   y[r]  = W x[r]                       experts   y[r]  = W_e x[r]
    data     dx[r] = W_e^T dy[r]                  weights   dW_e  = sum over the rows r of e of dy[r] x[r]^T  (fp32)
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TILE = 128


def case(name, op, dtype, rows, n, k, group=128, experts=1, active=1):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "n": n, "k": k, "group": group, "experts": experts,
            "active": active}


def listed():
    return [
        # one token through a small projection: nothing but latency
        case("matvec_1x1024x1024_bf16", "matvec", "bf16", 1, 1024, 1024),
        # one token through a large layer, finer scales
        case("matvec_1x8192x8192_bf16", "matvec", "bf16", 1, 8192, 8192, 64),
        # three sequences in full precision, a feature count and a reduction that fill no tile
        case("matvec_3x4097x1000_fp32", "matvec", "fp32", 3, 4097, 1000, 32),
        # a small batch of sequences through the widest layer
        case("matvec_16x16384x8192_fp16", "matvec", "fp16", 16, 16384, 8192),
        # one decoding step of 8 sequences, two experts of 64 each: most experts have no row
        case("experts_16x2048x2048_bf16", "experts", "bf16", 16, 2048, 2048, 64, 64, 13),
        # a short prompt, odd sizes, two experts without rows, full precision
        case("experts_301x777x1000_fp32", "experts", "fp32", 301, 777, 1000, 32, 7, 5),
        # a larger decoding batch: some 32 rows for each of 32 experts
        case("experts_1024x2048x4096_fp16", "experts", "fp16", 1024, 2048, 4096, 128, 32, 32),
        # long prompts: some 2048 rows for each of 8 experts
        case("experts_16384x4096x4096_bf16", "experts", "bf16", 16384, 4096, 4096, 128, 8, 8),
        # a training step's gradient with respect to the experts' inputs
        case("data_4096x4096x4096_bf16", "data", "bf16", 4096, 4096, 4096, 128, 8, 8),
        # the same at odd sizes, with an expert that got nothing
        case("data_333x1000x777_fp16", "data", "fp16", 333, 1000, 777, 64, 5, 4),
        # a training step's gradient with respect to the experts' weights
        case("weights_4096x2048x4096_bf16", "weights", "bf16", 4096, 2048, 4096, 128, 8, 8),
        # the same at odd sizes in full precision, with an expert that got nothing
        case("weights_500x513x1000_fp32", "weights", "fp32", 500, 513, 1000, 32, 6, 5),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if v >= 64 and rng.random() < 0.5:
            v = (v + 31) // 64 * 64
        return max(lo, min(hi, v))

    while True:
        op = rng.choice(["matvec", "experts", "data", "weights"])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        n, k, group = size(64, 16384), size(64, 8192), rng.choice([32, 64, 128])
        if op == "matvec":
            return {"op": op, "dtype": dtype, "rows": rng.choice([1, 1, 2, 3, 4, 7, 8, 13, 16]), "n": n, "k": k,
                    "group": group, "experts": 1, "active": 1}
        experts = size(1, 64)
        rows = size(1, 16384)
        active = min(rows, rng.choice([experts, rng.randint(max(1, experts // 2), experts)]))
        if experts * n * k <= 1 << 27 and rows * n * k <= 1 << 37:
            return {"op": op, "dtype": dtype, "rows": rows, "n": n, "k": k, "group": group, "experts": experts,
                    "active": active}


def padded(v):
    return (v + TILE - 1) // TILE * TILE


def quantize(w, group):
    """fp32 [n][k] -> (codes of one matrix, scales, alpha) in the layout above."""
    n, k = w.shape
    full = torch.zeros((padded(n), padded(k)), dtype=torch.float32, device=w.device)
    full[:n, :k] = w
    alpha = full.abs().amax() / (15.0 * 448.0)
    groups = full.view(padded(n), -1, group)
    scale = (groups.abs().amax(2) / (15.0 * alpha)).clamp_(max=448.0).to(torch.float8_e4m3fn)
    step = alpha * scale.float()
    t = torch.where(step.unsqueeze(2) > 0, groups / step.clamp_min(1e-30).unsqueeze(2), torch.zeros_like(groups))
    t = ((t + 15.0) / 2.0).round_().clamp_(0, 15).to(torch.int32)
    #              tile_n       row   tile_k            w  c  p  h
    t = t.view(padded(n) // TILE, TILE, padded(k) // TILE, 4, 4, 4, 2)
    shift = (4 * torch.arange(4, device=w.device).view(4, 1) + 16 * torch.arange(2, device=w.device)).to(torch.int32)
    words = (t << shift).sum((5, 6)).to(torch.int32).permute(0, 2, 4, 1, 3).contiguous()
    scales = scale.view(torch.uint8).view(padded(n) // TILE, TILE, padded(k) // TILE, TILE // group)
    return words, scales.permute(0, 2, 3, 1).contiguous(), alpha


def row_counts(case, seed):
    """Rows of each expert: `active` of them have at least one, the others none; some are asked for more than others."""
    rng = np.random.default_rng(seed)
    counts = np.zeros(case["experts"], dtype=np.int64)
    chosen = rng.choice(case["experts"], case["active"], replace=False)
    counts[chosen] = 1
    share = rng.uniform(0.5, 1.5, case["active"])
    counts[chosen] += rng.multinomial(case["rows"] - case["active"], share / share.sum())
    return counts


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    experts, rows, n, k, group = (case[key] for key in ("experts", "rows", "n", "k", "group"))
    counts = row_counts(case, seed)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    state = dict(case, dtype=dtype, offsets=torch.tensor(offsets, dtype=torch.int32, device=dev),
                 longest=int(counts.max()))                # the buffer capacity that a padding program keeps
    if case["op"] != "weights":
        shape = (experts, padded(n) // TILE, padded(k) // TILE)
        state["codes"] = torch.empty(shape + (4, TILE, 4), dtype=torch.int32, device=dev)
        state["scales"] = torch.empty(shape + (TILE // group, TILE), dtype=torch.uint8, device=dev)
        state["alpha"] = torch.empty(experts, dtype=torch.float32, device=dev)
        for e in range(experts):
            w = torch.randn((n, k), generator=gen, device=dev) / math.sqrt(k)
            state["codes"][e], state["scales"][e], state["alpha"][e] = quantize(w, group)
    if case["op"] != "data":
        # activations: most channels of unit size, a few much larger
        size = 1.0 + 7.0 * (torch.rand(k, generator=gen, device=dev) < 0.01)
        state["x"] = (torch.randn((rows, k), generator=gen, device=dev) * size).to(dtype)
    if case["op"] in ("data", "weights"):
        state["dy"] = (torch.randn((rows, n), generator=gen, device=dev) * 0.05).to(dtype)
    return state


def decoded(state):
    """fp32 [experts][n][k] of the stored weights."""
    codes, scales, group = state["codes"], state["scales"], state["group"]
    experts, tn, tk = codes.shape[:3]
    bit = torch.arange(8, dtype=torch.int32, device=codes.device)
    bit = (bit // 2) * 4 + (bit % 2) * 16
    t = (codes.unsqueeze(-1) >> bit) & 15                                      # [experts][tn][tk][c][row][w][j]
    q = (2 * t - 15).to(torch.float32).permute(0, 1, 4, 2, 5, 3, 6)             # [experts][tn][row][tk][w][c][j]
    s = scales.view(torch.float8_e4m3fn).to(torch.float32).permute(0, 1, 4, 2, 3)   # [experts][tn][row][tk][groups]
    w = q.reshape(experts, tn, TILE, tk, TILE // group, group) * s.unsqueeze(-1)
    w = w.reshape(experts, tn * TILE, tk * TILE)[:, :state["n"], :state["k"]]
    return w * state["alpha"].view(-1, 1, 1)


def run(state):
    if own:
        return run_own(state)
    op, dtype = state["op"], state["dtype"]
    if op == "matvec":
        return torch.matmul(state["x"].float(), decoded(state)[0].t()).to(dtype)
    # rows into a padded [experts][longest][.] array, one batched product, and back
    offsets = state["offsets"]
    row = torch.arange(state["rows"], device=offsets.device, dtype=torch.int32)
    expert = (row.view(-1, 1) >= offsets[1:].view(1, -1)).sum(1)
    place = row - offsets[expert]

    def spread(v):
        full = torch.zeros((state["experts"], state["longest"], v.shape[1]), dtype=torch.float32, device=v.device)
        full[expert, place] = v.float()
        return full

    if op == "experts":
        return torch.matmul(spread(state["x"]), decoded(state).transpose(1, 2))[expert, place].to(dtype)
    if op == "data":
        return torch.matmul(spread(state["dy"]), decoded(state))[expert, place].to(dtype)
    return torch.matmul(spread(state["dy"]).transpose(1, 2), spread(state["x"]))


def run_own(state):
    from paper_2106_09886_b200 import qnn
    op = state["op"]
    if op == "weights":
        return qnn.expert_gemm_backward_weights(state["dy"], state["x"], state["offsets"])
    w = qnn.G4Weights(state["codes"], state["scales"], state["alpha"], state["n"], state["k"], state["group"])
    if op == "matvec":
        return qnn.g4_matvec(state["x"], w)
    if op == "experts":
        return qnn.g4_expert_gemm(state["x"], w, state["offsets"])
    return qnn.g4_expert_gemm_backward_data(state["dy"], w, state["offsets"])


def exact(case, seed):
    state = prepare(case, seed)
    n, k, group, op = state["n"], state["k"], state["group"], state["op"]
    dev = state["offsets"].device
    bounds = state["offsets"].tolist()
    if op != "weights":
        # element (row, col) looked up by its address
        col = torch.arange(k, device=dev)
        row = torch.arange(n, device=dev)
        tk = padded(k) // TILE
        inner = col % TILE
        at_col = (col // TILE) * 2048 + (inner // 8 % 4) * 512 + inner // 32
        at_row = (row // TILE) * tk * 2048 + (row % TILE) * 4
        bits = (inner % 8 // 2) * 4 + (inner % 2) * 16
        s_col = (col // TILE) * (TILE * TILE // group) + (inner // group) * TILE
        s_row = (row // TILE) * tk * (TILE * TILE // group) + row % TILE
        byte = torch.arange(256, device=dev)
        exponent, mantissa = (byte // 8 % 16).double(), (byte % 8).double()
        table = torch.where(exponent > 0, (8 + mantissa) * torch.exp2(exponent - 10), mantissa * 2.0 ** -9)

    def weights_of(e):
        word = state["codes"][e].reshape(-1)[at_row.view(-1, 1) + at_col]
        code = torch.bitwise_and(torch.bitwise_right_shift(word, bits), 15).double()
        scale = table[state["scales"][e].reshape(-1)[s_row.view(-1, 1) + s_col].long()]
        return (code + code - 15.0) * scale * state["alpha"][e].double()

    if op == "matvec":
        return state["x"].double() @ weights_of(0).t()
    if op == "weights":
        out = torch.zeros((state["experts"], n, k), dtype=torch.float64, device=dev)
    else:
        out = torch.zeros((state["rows"], n if op == "experts" else k), dtype=torch.float64, device=dev)
    for e in range(state["experts"]):
        a, b = bounds[e], bounds[e + 1]
        if a == b:
            continue
        if op == "experts":
            out[a:b] = state["x"][a:b].double() @ weights_of(e).t()
        elif op == "data":
            out[a:b] = state["dy"][a:b].double() @ weights_of(e)
        else:
            out[e] = state["dy"][a:b].double().t() @ state["x"][a:b].double()
    return out


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    rows, n, k = case["rows"], case["n"], case["k"]
    matrix = n * k // 2 + n * (-(-k // case["group"])) + 4          # codes, scales and alpha of one expert
    if case["op"] == "weights":
        moved = rows * (n + k) * size + case["experts"] * n * k * 4
    else:
        moved = rows * (n + k) * size + case["active"] * matrix
    return {"bytes": moved + 4 * (case["experts"] + 1) * (case["op"] != "matvec"), "flops": 2 * rows * n * k}

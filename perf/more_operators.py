"""Timed cases of routing to experts, root-mean-square norm with a residual and 8-bit output, and products in 8-bit integers.

    route    per token the `top` experts of `experts` by score (softmax or sigmoid of the logits), a bias added for the choice
             alone, the choice limited to `top_groups` of `groups` equal groups; weights from the unbiased scores; and the plan
             that grouped products go by: order (the slot token * top + choice of each row, rows sorted by expert, slots in
             order within one), place (the row of each slot) and offsets (an expert's first row)
    gates    the gradient of the weights with respect to the logits
    norm     h = x + residual, rounded to its type;  y = h / sqrt(mean h^2 + eps) * gain, as real numbers or in 8 bits with a
             scale for each row: scale = max(max|y| / 127, 2^-126), code = y / scale to nearest
    normgrad its backward products
    product  y[r][j] = scale[r] * scale[j] * sum_i x[r][i] w[j][i] on 8-bit codes, of rows in 8 bits or of real rows
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
SMALLEST = 2.0 ** -126
EPS = 1e-6


def route(name, op, dtype, tokens, experts, top, score="softmax", bias=False, groups=1, top_groups=1, group_score="max",
          renormalise=True, factor=1.0, padded=0):
    return {"name": name, "op": op, "dtype": dtype, "tokens": tokens, "experts": experts, "top": top, "score": score, "bias": bias,
            "groups": groups, "top_groups": top_groups, "group_score": group_score, "renormalise": renormalise, "factor": factor,
            "padded": padded}


def norm(name, op, dtype, rows, width, residual=True, eight=False):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "width": width, "residual": residual, "eight": eight}


def product(name, dtype, rows, n, k, real=False, bias=False):
    return {"name": name, "op": "product", "dtype": dtype, "rows": rows, "n": n, "k": k, "real": real, "bias": bias}


def listed():
    return [
        # one token of a decoding step: nothing but latency
        route("route_1x64_top6_bf16", "route", "bf16", 1, 64, 6),
        # a small layer's batch, two of eight experts
        route("route_512x8_top2_fp32", "route", "fp32", 512, 8, 2),
        # long prompts through many experts in groups, balanced by a bias
        route("route_16384x256_top8_fp32", "route", "fp32", 16384, 256, 8, "sigmoid", True, 8, 4, "top2", True, 2.5),
        # a training step's gradient of scores that are not renormalised, odd sizes, some tokens padding
        route("gates_4097x160_top6_fp32", "gates", "fp32", 4097, 160, 6, renormalise=False, padded=61),
        # a decoding step's token, with its residual, into 8 bits
        norm("norm_1x4096_8bit_bf16", "norm", "bf16", 1, 4096, True, True),
        # prompts into 8 bits
        norm("norm_16384x4096_8bit_bf16", "norm", "bf16", 16384, 4096, True, True),
        # a width that fills no vector, real output, no residual
        norm("norm_777x1001_fp16", "norm", "fp16", 777, 1001, False, False),
        # a training step's gradients
        norm("normgrad_8192x4096_bf16", "normgrad", "bf16", 8192, 4096),
        # one token through a large layer
        product("product_1x8192x8192_bf16", "bf16", 1, 8192, 8192),
        # a decoding step of 16 sequences through the widest layer
        product("product_16x16384x8192_fp16", "fp16", 16, 16384, 8192),
        # a short prompt of real rows, odd sizes, full precision out
        product("product_301x777x1001_real_fp32", "fp32", 301, 777, 1001, True, True),
        # long prompts
        product("product_8192x8192x8192_bf16", "bf16", 8192, 8192, 8192),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if v >= 64 and rng.random() < 0.5:
            v = (v + 31) // 64 * 64
        return max(lo, min(hi, v))

    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    op = rng.choice(["route", "route", "gates", "norm", "norm", "normgrad", "product", "product", "product"])
    if op in ("route", "gates"):
        tokens, groups = size(1, 16384), rng.choice([1, 1, 2, 4, 8])
        each = size(2, 256 // groups)
        if groups == 1:
            each = max(each, 4)
        top_groups = rng.randint(1, groups)
        top = rng.randint(1, min(8, each * top_groups))
        score, bias = rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5
        case = route("", op, rng.choice(["fp32", dtype]), tokens, groups * each, top, score, bias, groups, top_groups,
                     rng.choice(["max", "top2"]), rng.random() < 0.5, rng.choice([1.0, 2.5]),
                     rng.choice([0, 0, tokens // 7]))
    elif op == "product":
        while True:
            rows, n, k = rng.choice([1, 2, 5, 8, 16, 32, size(1, 8192), size(1, 8192)]), size(64, 16384), size(64, 16384)
            if rows * n * k <= 1 << 39 and n * k <= 1 << 27:
                break
        case = product("", dtype, rows, n, k, rng.random() < 0.3, rng.random() < 0.3)
    else:
        while True:
            rows, width = size(1, 16384), size(64, 16384)
            if rows * width * BYTES[dtype] <= 1 << 27:
                break
        case = norm("", op, dtype, rows, width, rng.random() < 0.7, op == "norm" and rng.random() < 0.6)
    del case["name"]
    return case


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype, op = TYPES[case["dtype"]], case["op"]
    state = dict(case, dtype=dtype)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def codes(rows, k):
        # rows lie a multiple of 16 bytes apart, as the framework's calls lay them out
        full = torch.zeros((rows, (k + 15) // 16 * 16), dtype=torch.int8, device=dev)
        full[:, :k] = (normal(rows, k) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
        return full[:, :k]

    if op in ("route", "gates"):
        tokens, experts = case["tokens"], case["experts"]
        # some experts are asked for more than others
        state["logits"] = (normal(tokens, experts) * 1.5 + 0.5 * normal(experts)).to(dtype)
        state["bias"] = normal(experts) * 0.05 if case["bias"] else None
        state["mask"] = None
        if case["padded"]:
            state["mask"] = torch.ones(tokens, dtype=torch.bool, device=dev)
            state["mask"][torch.randperm(tokens, generator=gen, device=dev)[:case["padded"]]] = False
        if op == "gates":
            state["chosen"] = choose(state)[0]
            state["dweights"] = normal(tokens, case["top"]) * 0.1
    elif op == "product":
        rows, n, k = case["rows"], case["n"], case["k"]
        state["w"], state["w_scales"] = codes(n, k), (0.5 + torch.rand(n, generator=gen, device=dev)) * 1e-3
        if case["real"]:
            state["x"] = normal(rows, k).to(dtype)
        else:
            state["x"], state["x_scales"] = codes(rows, k), (0.5 + torch.rand(rows, generator=gen, device=dev)) * 0.02
        state["bias"] = normal(n) if case["bias"] else None
    else:
        rows, width = case["rows"], case["width"]
        # most channels of unit size, a few much larger
        size = 1.0 + 7.0 * (torch.rand(width, generator=gen, device=dev) < 0.01)
        state["gain"] = (1.0 + 0.2 * normal(width)).to(dtype)
        if op == "norm":
            state["x"] = (normal(rows, width) * size).to(dtype)
            state["residual"] = (normal(rows, width) * size).to(dtype) if case["residual"] else None
        else:
            h = (normal(rows, width) * size).to(dtype)
            state["h"], state["dy"] = h, (normal(rows, width) * 0.05).to(dtype)
            state["rstd"] = torch.rsqrt(h.double().square().mean(1) + EPS).float()
            state["dh"] = (normal(rows, width) * 0.05).to(dtype) if case["residual"] else None
    return state


def scores(logits, kind):
    if kind == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def choose(state):
    """(experts, scores) of the choice; in 64 bits, for keys that lie next to one another."""
    logits, bias = state["logits"].double(), state["bias"]
    tokens, experts = logits.shape
    score = scores(logits, state["score"])
    if bias is None and (state["groups"] == 1 or state["group_score"] == "max"):
        key = logits                                               # scores grow with the logits
    else:
        key = score if bias is None else score + bias.double()
    allowed = key
    if state["groups"] > 1:
        each = key.view(tokens, state["groups"], -1)
        if state["group_score"] == "max":
            best = each.amax(2)
        else:
            best = each.sort(2, descending=True).values[:, :, :2].sum(2)
        keep = best.sort(dim=1, descending=True, stable=True).indices[:, :state["top_groups"]]
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, keep, True)
        order_by = logits if bias is None else key                 # (sums of two scores decide between groups alone)
        allowed = torch.where(kept.unsqueeze(2), order_by.view(each.shape), -math.inf).view(tokens, experts)
    chosen = allowed.sort(dim=1, descending=True, stable=True).indices[:, :state["top"]]
    score = score.gather(1, chosen)
    if state["mask"] is not None:
        chosen = torch.where(state["mask"].view(-1, 1), chosen, -1)
        score = torch.where(state["mask"].view(-1, 1), score, 0.0)
    return chosen.to(torch.int32), score


def run_route(state):
    chosen, score = choose(state)
    total = score.sum(1, keepdim=True) if state["renormalise"] else torch.ones_like(score[:, :1])
    weights = torch.where(chosen >= 0, score / torch.where(total > 0, total, 1.0) * state["factor"], 0.0).float()
    experts = state["experts"]
    flat = chosen.reshape(-1).long()
    flat = torch.where(flat < 0, experts, flat)
    order = flat.sort(stable=True).indices
    offsets = torch.zeros(experts + 2, dtype=torch.int32, device=flat.device)
    offsets[1:] = torch.zeros(experts + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, flat, torch.ones_like(flat)).cumsum(0)
    offsets = offsets[:experts + 1].contiguous()
    row = torch.arange(flat.numel(), device=flat.device)
    there = row < offsets[-1]
    place = torch.empty_like(flat).scatter_(0, order, torch.where(there, row, -1))
    order = torch.where(there, order, -1)
    return {"experts": chosen, "weights": weights, "order": order.to(torch.int32), "place": place.view(chosen.shape).to(torch.int32),
            "offsets": offsets}


def run_gates(state):
    logits, chosen, dw = state["logits"].float(), state["chosen"].long(), state["dweights"]
    there = chosen >= 0
    at = chosen.clamp_min(0)
    score = scores(logits, state["score"])
    s = torch.where(there, score.gather(1, at), 0.0)
    dw = torch.where(there, dw, 0.0) * state["factor"]
    if state["renormalise"]:
        total = s.sum(1, keepdim=True)
        total = torch.where(total > 0, total, 1.0)
        ds = (dw - (dw * s).sum(1, keepdim=True) / total) / total
    else:
        ds = dw
    out = torch.zeros_like(logits)
    if state["score"] == "sigmoid":
        return out.scatter_add_(1, at, torch.where(there, ds * s * (1.0 - s), 0.0)).to(state["dtype"])
    out.scatter_add_(1, at, torch.where(there, ds, 0.0))
    if not state["renormalise"]:
        out = out - (ds * s).sum(1, keepdim=True)                  # (renormalised, this sum is zero)
    return (out * score).to(state["dtype"])


def to_codes(y):
    """fp32 [rows][.] -> (whole numbers as fp32, scales)."""
    scale = (y.abs().amax(1) / torch.full((), 127.0, device=y.device)).clamp_min(SMALLEST)
    return (y / scale.view(-1, 1)).round().clamp(-127, 127), scale


def run_norm(state):
    h = state["x"]
    if state["residual"] is not None:
        h = (h.float() + state["residual"].float()).to(state["dtype"])
    v = h.float()
    rstd = torch.rsqrt(v.square().mean(1) + EPS)
    y = v * rstd.view(-1, 1) * state["gain"].float()
    out = {"rstd": rstd}
    if state["residual"] is not None:
        out["h"] = h
    if state["eight"]:
        codes, scale = to_codes(y)
        out["values"] = (codes * scale.view(-1, 1)).to(torch.float16 if state["dtype"] == torch.float16 else torch.bfloat16)
        out["scales"] = scale
    else:
        out["y"] = y.to(state["dtype"])
    return out


def run_normgrad(state):
    h, dy, rstd = state["h"].float(), state["dy"].float(), state["rstd"].view(-1, 1)
    unit = h * rstd
    a = dy * state["gain"].float()
    dx = (a - unit * (a * unit).mean(1, keepdim=True)) * rstd
    if state["dh"] is not None:
        dx = dx + state["dh"].float()
    return {"dx": dx.to(state["dtype"]), "dgain": (dy * unit).sum(0)}


def run_product(state):
    if state["real"]:
        x, scale = to_codes(state["x"].float())
    else:
        x, scale = state["x"].float(), state["x_scales"]
    y = torch.matmul(x, state["w"].float().t()) * scale.view(-1, 1) * state["w_scales"]
    if state["bias"] is not None:
        y = y + state["bias"]
    return y.to(state["dtype"])


def run(state):
    if own:
        return run_own(state)
    return {"route": run_route, "gates": run_gates, "norm": run_norm, "normgrad": run_normgrad, "product": run_product}[state["op"]](state)


def run_own(state):
    from paper_2106_09886_b200 import qnn
    op = state["op"]
    if op == "route":
        r = qnn.route(state["logits"], state["top"], state["score"], state["bias"], state["groups"], state["top_groups"],
                      state["group_score"], state["renormalise"], state["factor"], state["mask"])
        return {"experts": r.experts, "weights": r.weights, "order": r.order, "place": r.place, "offsets": r.offsets}
    if op == "gates":
        return qnn.route_backward(state["dweights"], state["logits"], state["chosen"], state["score"], state["renormalise"],
                                  state["factor"])
    if op == "normgrad":
        dx, dgain = qnn.rms_norm_backward(state["dy"], state["h"], state["gain"], state["rstd"], state["dh"])
        return {"dx": dx, "dgain": dgain}
    if op == "norm":
        if state["eight"]:
            rows, h, rstd = qnn.rms_norm_i8(state["x"], state["gain"], EPS, state["residual"])
            kind = torch.float16 if state["dtype"] == torch.float16 else torch.bfloat16
            out = {"values": qnn.i8_decode(rows, kind), "scales": rows.scales}
        else:
            y, h, rstd = qnn.rms_norm(state["x"], state["gain"], EPS, state["residual"])
            out = {"y": y}
        out["rstd"] = rstd
        if state["residual"] is not None:
            out["h"] = h
        return out
    x = qnn.i8_quantize(state["x"]) if state["real"] else qnn.I8Rows(state["x"], state["x_scales"])
    return qnn.i8_gemm(x, qnn.I8Rows(state["w"], state["w_scales"]), state["dtype"], state["bias"])


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("route", "gates"):
        logits = state["logits"].double()
        if case["score"] == "softmax":
            p = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))
        else:
            p = torch.where(logits < 0, torch.exp(logits) / (torch.exp(logits) + 1.0), 1.0 / (torch.exp(-logits) + 1.0))
        if op == "route":
            # the largest that is left, `top` times (first of the groups, then of their experts)
            left = logits.clone() if state["bias"] is None else p + state["bias"].double()
            if case["groups"] > 1:
                by_sums = case["group_score"] == "top2"
                sides = (p if state["bias"] is None and by_sums else left).unflatten(1, (case["groups"], -1))
                worth = sides.topk(2, 2).values.sum(2) if by_sums else sides.max(2).values
                open_ = torch.zeros_like(worth)
                for _ in range(case["top_groups"]):
                    g = worth.argmax(1, keepdim=True)
                    open_.scatter_(1, g, 1.0)
                    worth.scatter_(1, g, -math.inf)
                left = left.masked_fill(open_.repeat_interleave(left.shape[1] // case["groups"], 1) == 0, -math.inf)
            picks = []
            for _ in range(case["top"]):
                picks.append(left.argmax(1, keepdim=True))
                left.scatter_(1, picks[-1], -math.inf)
            chosen = torch.cat(picks, 1)
            if state["mask"] is not None:
                chosen[~state["mask"]] = -1
        else:
            chosen, dw = state["chosen"].long(), state["dweights"].double()
        there, at = chosen >= 0, chosen.clamp_min(0)
        hit = torch.zeros((case["tokens"], case["top"], case["experts"]), dtype=torch.bool, device=logits.device)
        if hit.numel() > 1 << 27:
            return None
        hit.scatter_(2, at.unsqueeze(2), there.unsqueeze(2))
        s = (p.unsqueeze(1) * hit).sum(2)                          # 0 where there is none
        total = s.sum(1, keepdim=True).clamp_min(1e-300)
        if op == "route":
            w = case["factor"] * (s / total if case["renormalise"] else s)
            return {"experts": None, "weights": w, "order": None, "place": None, "offsets": None}
        # d weight_i / d score_j, then d score_j / d logit_m
        dw = dw * there * case["factor"]
        ds = dw if not case["renormalise"] else dw / total - (dw * s).sum(1, keepdim=True) / total ** 2
        dp = (ds.unsqueeze(2) * hit).sum(1)
        if case["score"] == "sigmoid":
            return dp * p * (1.0 - p)
        return p * dp - p * (p * dp).sum(1, keepdim=True)
    if op == "norm":
        h = state["x"].double()
        if case["residual"]:
            h = (h + state["residual"].double()).to(state["dtype"]).double()
        rstd = (h.pow(2).sum(1) / case["width"] + EPS).pow(-0.5)
        y = h * rstd[:, None] * state["gain"].double()
        out = {"rstd": rstd}
        if case["residual"]:
            out["h"] = h
        if case["eight"]:
            scale = torch.maximum(y.abs().amax(1) / 127.0, torch.full((), SMALLEST, dtype=torch.float64, device=y.device))
            out["values"], out["scales"] = torch.clamp(torch.round(y / scale[:, None]), -127, 127) * scale[:, None], scale
        else:
            out["y"] = y
        return out
    if op == "normgrad":
        h, dy, r, g = state["h"].double(), state["dy"].double(), state["rstd"].double()[:, None], state["gain"].double()
        inner = (h * dy * g).sum(1, keepdim=True)
        dx = dy * g * r - h * r ** 3 * inner / case["width"]
        if state["dh"] is not None:
            dx = dx + state["dh"].double()
        return {"dx": dx, "dgain": (h * dy * r).sum(0)}
    if case["real"]:
        x = state["x"].double()
        scale = (x.abs().amax(1) / 127.0).clamp_min(SMALLEST).float().double()
        x = torch.clamp(torch.round((x / scale[:, None]).float()), -127, 127).double()
    else:
        x, scale = state["x"].double(), state["x_scales"].double()
    y = x @ state["w"].double().t() * (scale[:, None] * state["w_scales"].double())
    return y if state["bias"] is None else y + state["bias"].double()


def work(case):
    op, size = case["op"], BYTES[case["dtype"]]
    if op in ("route", "gates"):
        tokens, experts, top = case["tokens"], case["experts"], case["top"]
        if op == "route":
            moved = tokens * (experts * size + top * 16 + (1 if case["padded"] else 0)) + 4 * (experts + 1) + (4 * experts if case["bias"] else 0)
        else:
            read = experts if case["score"] == "softmax" and not case["renormalise"] else top
            moved = tokens * ((read + experts) * size + top * 8)
        return {"bytes": moved, "flops": tokens * experts * 4}
    if op == "product":
        rows, n, k = case["rows"], case["n"], case["k"]
        x = rows * k * size if case["real"] else rows * (k + 4)
        return {"bytes": x + n * (k + 4) + (4 * n if case["bias"] else 0) + rows * n * size, "flops": 2 * rows * n * k}
    rows, width = case["rows"], case["width"]
    if op == "normgrad":
        return {"bytes": rows * (width * size * (4 if case["residual"] else 3) + 4) + width * (size + 4), "flops": 9 * rows * width}
    out = 3 if case["eight"] else size                             # codes and the values that they stand for
    return {"bytes": rows * (width * (size * (3 if case["residual"] else 1) + out) + 8) + width * size, "flops": 8 * rows * width}

"""Run one library call on synthetic device data a few times and print its timing (one JSON line).

    python -m paper_2106_09886_b200.run_case gemm   --m 4096 --n 4096 --k 4096 --ab 2 --wb 2 [--reps 5]
    python -m paper_2106_09886_b200.run_case conv   --N 32 --H 14 --W 14 --C 256 --Cout 256 --R 3 --S 3 --stride 1 --pad 1 --ab 2 --wb 2
    python -m paper_2106_09886_b200.run_case encode --rows 4096 --k 4096 --bits 2
    python -m paper_2106_09886_b200.run_case backward_conv --N 32 --H 14 --W 14 --C 256 --Cout 256
    python -m paper_2106_09886_b200.run_case stack  --net vgg16 [--batch 64] [--layers 0,1] [--table]
    python -m paper_2106_09886_b200.run_case experts --tokens 512 --experts 8 --top 2 --hidden 1024 --inner 2048
    python -m paper_2106_09886_b200.run_case block  --tokens 512 --experts 32 --top 4 --groups 4 --hidden 1024 --inner 512

Inputs are drawn on the device (half-normal activations, normal weights); this is a timing and
profiling driver, correctness is the business of the test-suite.  Times are CUDA-event times of
the single library call, after `--warmup` untimed calls, rotating over `--sets` input/output sets
so that consecutive calls do not find their data in L2.
"""
from __future__ import annotations

import argparse
import json
import statistics

import torch

from . import qnn


_flush_buf = None


def flush_l2():
    """Writes a buffer twice the size of the L2 cache, so that the next call finds none of its data there."""
    global _flush_buf
    if _flush_buf is None:
        _flush_buf = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    _flush_buf.zero_()


def _time_calls(fn, reps: int, warmup: int, flush: bool = False):
    for i in range(warmup):
        fn(i)
    torch.cuda.synchronize()
    times = []
    for i in range(reps):
        if flush:
            flush_l2()
        else:
            torch.cuda._sleep(60000)      # keeps the GPU busy (~30 us) while the host enqueues, so that the event pair
                                          # brackets the kernel and not the host's launch latency
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        fn(i)
        e1.record()
        e1.synchronize()
        times.append(e0.elapsed_time(e1))
    return times


def layer_roofline(Mg, Ng, ab, wb, conv, R, S, C, in_rows, ms, popc_per_s, hbm_gbs):
    """Roofline of one contraction launch: the slower of its algorithmic bytes at the HBM peak (packed activations of
    the `in_rows` input rows or pixels and packed weights read once, fp32 outputs written once) and its popcount
    instructions at the measured popcount rate (the scarce pipe; qnn_popcounts_per_output per output element)."""
    kg = R * S * C
    nbytes = in_rows * C * ab / 8.0 + Ng * kg * wb / 8.0 + Mg * Ng * 4.0
    popc = qnn.popcounts_per_output(ab, wb, conv, R, S, C, Ng)
    t_alu = Mg * Ng * popc / popc_per_s * 1e3
    t_hbm = nbytes / (hbm_gbs * 1e9) * 1e3
    bound = "alu" if t_alu >= t_hbm else "hbm"
    binary = 2.0 * Mg * Ng * kg * ab * wb
    if bound == "alu":
        achieved, peak, unit = binary / (ms * 1e-3) / 1e12, binary / (t_alu * 1e-3) / 1e12, "binary TOPS"
    else:
        achieved, peak, unit = nbytes / (ms * 1e-3) / 1e9, hbm_gbs, "GB/s"
    return {"bound": bound, "achieved": achieved, "peak": peak, "unit": unit, "frac": max(t_alu, t_hbm) / ms,
            "roofline_ms": max(t_alu, t_hbm), "popc_per_word": popc / (ab * wb * (kg / 32.0)), "alg_bytes": nbytes}


def time_gemm(Mg, Ng, Kg, ab, wb, reps=5, warmup=3, sets=3, dev="cuda:0", seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    w = torch.randn((Ng, Kg), device=dev, generator=g) * 0.02
    sw = float(w.abs().max()) / (2 ** wb - 1)
    packed = qnn.pack_weights(w, Ng, 1, Kg, qnn.W_NTC, wb, sw)
    planes, outs = [], []
    for _ in range(sets):
        a = torch.randn((Mg, Kg), device=dev, generator=g).abs_().clamp_(max=4.0)
        planes.append(qnn.encode_pack(a, ab, 4.0 / (2 ** ab - 1)))
        outs.append(torch.empty((Mg, Ng), dtype=torch.float32, device=dev))
        del a
    times = _time_calls(lambda i: qnn.bgemm(planes[i % sets], ab, packed, wb, Mg, Ng, Kg, 1e-3, out=outs[i % sets]),
                        reps, warmup)
    return _report("qnn_bgemm", Mg, Ng, Kg, ab, wb, times)


def time_conv(N, H, W, C, Cout, R, S, stride, pad, ab, wb, reps=5, warmup=3, sets=2, dev="cuda:0", seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    w = torch.randn((Cout, R, S, C), device=dev, generator=g) * 0.02
    sw = float(w.abs().max()) / (2 ** wb - 1)
    packed = qnn.pack_weights(w, Cout, R * S, C, qnn.W_NTC, wb, sw)
    Ho, Wo = qnn.conv_out_dim(H, R, stride, pad), qnn.conv_out_dim(W, S, stride, pad)
    planes, outs = [], []
    for _ in range(sets):
        a = torch.randn((N * H * W, C), device=dev, generator=g).clamp_(min=0.0)
        planes.append(qnn.encode_pack(a, ab, 4.0 / (2 ** ab - 1)))
        outs.append(torch.empty((N, Ho, Wo, Cout), dtype=torch.float32, device=dev))
        del a
    times = _time_calls(lambda i: qnn.bconv2d(planes[i % sets], ab, packed, wb, N, H, W, C, Cout, R, S, stride, pad,
                                              1e-3, out=outs[i % sets]), reps, warmup)
    return _report("qnn_bconv2d", N * Ho * Wo, Cout, R * S * C, ab, wb, times)


def time_encode(rows, k, bits, reps=5, warmup=3, sets=3, relu=False, dev="cuda:0", seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    xs = [torch.randn((rows, k), device=dev, generator=g) for _ in range(sets)]
    planes = [torch.empty((rows, bits, qnn.row_words(k)), dtype=torch.int32, device=dev) for _ in range(sets)]
    times = _time_calls(lambda i: qnn.encode_pack(xs[i % sets], bits, 0.37, qnn.RELU if relu else 0,
                                                  planes=planes[i % sets]), reps, warmup)
    ms = statistics.median(times)
    nbytes = rows * k * 4 + rows * bits * qnn.row_words(k) * 4
    return {"call": "qnn_encode_pack", "rows": rows, "k": k, "bits": bits, "ms_median": ms, "ms_min": min(times),
            "bytes": nbytes, "gbs": nbytes / (ms * 1e-3) / 1e9}


def time_stack(net: str, batch: int, reps=3, warmup=2, dev="cuda:0", seed=0, layers=None):
    """Every quantized convolution of a ResNet-18- or VGG-16-shaped stack, each on its own synthetic
    input of the right shape (post-ReLU half-normal), timed as qnn_encode_pack + qnn_bconv2d."""
    from . import workloads as wl
    if net == "resnet18":
        shapes = wl.resnet18_shapes(batch)
    elif net in ("resnet18_p1", "resnet18_p2"):
        shapes = wl.resnet18_mixed_shapes(int(net[-1]), batch)     # Table 4's mixed precisions
    else:
        shapes = wl.vgg16_shapes(batch)
    g = torch.Generator(device=dev).manual_seed(seed)
    rows = []
    for li, s in enumerate(shapes):
        if layers is not None and li not in layers:
            continue
        w = torch.randn((s.Cout, s.R, s.S, s.C), device=dev, generator=g) * (2.0 / (s.R * s.S * s.C)) ** 0.5
        packed = qnn.pack_weights(w, s.Cout, s.R * s.S, s.C, qnn.W_NTC, s.wb, float(w.abs().max()) / (2 ** s.wb - 1))
        a = torch.randn((s.N * s.H * s.W, s.C), device=dev, generator=g)
        planes = torch.empty((s.N * s.H * s.W, s.ab, qnn.row_words(s.C)), dtype=torch.int32, device=dev)
        out = torch.empty((s.N, s.Ho, s.Wo, s.Cout), dtype=torch.float32, device=dev)
        sa = 4.0 / (2 ** s.ab - 1)
        t_enc = _time_calls(lambda i: qnn.encode_pack(a, s.ab, sa, qnn.RELU, planes=planes), reps, warmup)
        t_conv = _time_calls(lambda i: qnn.bconv2d(planes, s.ab, packed, s.wb, s.N, s.H, s.W, s.C, s.Cout, s.R, s.S,
                                                   s.stride, s.pad, 1e-3, out=out), reps, warmup)
        # layer chaining: the same convolution writing the next layer's planes instead of fp32
        nxt = torch.empty((s.Mg, s.ab, qnn.row_words(s.Cout)), dtype=torch.int32, device=dev)
        fused_out = out if (s.R * s.S * s.C <= 32) else None      # single-word patches encode from the fp32 result
        t_fused = _time_calls(lambda i: qnn.bconv2d_encode(planes, s.ab, packed, s.wb, s.N, s.H, s.W, s.C, s.Cout, s.R,
                                                           s.S, s.stride, s.pad, 1e-3, s.ab, sa, qnn.RELU,
                                                           next_planes=nxt, out=fused_out), reps, warmup)
        del nxt
        enc_ms, conv_ms = statistics.median(t_enc), statistics.median(t_conv)
        macs = float(s.Mg) * s.Cout * s.Kg
        rows.append({"layer": s.name, "Mg": s.Mg, "Ng": s.Cout, "Kg": s.Kg, "ab": s.ab, "wb": s.wb,
                     "R": s.R, "S": s.S, "C": s.C, "stride": s.stride, "in_rows": s.N * s.H * s.W,
                     "encode_ms": enc_ms, "conv_ms": conv_ms, "conv_encode_ms": statistics.median(t_fused),
                     "conv_binary_tops": 2 * macs * s.ab * s.wb / (conv_ms * 1e-3) / 1e12,
                     "conv_equiv_int_gops": 2 * macs / (conv_ms * 1e-3) / 1e9,
                     "encode_gbs": (a.numel() * 4 + planes.numel() * 4) / (enc_ms * 1e-3) / 1e9,
                     "out_bytes": out.numel() * 4, "in_bytes_fp32": a.numel() * 4, "int_macs": macs})
        del a, planes, out, w, packed
    tot_ms = sum(r["encode_ms"] + r["conv_ms"] for r in rows)
    tot_macs = sum(r["int_macs"] for r in rows)
    bin_macs = sum(r["int_macs"] * r["ab"] * r["wb"] for r in rows)
    return {"call": f"stack:{net}", "batch": batch, "layers": rows, "total_ms": tot_ms,
            "binary_tops": 2 * bin_macs / (tot_ms * 1e-3) / 1e12, "equiv_int_gops": 2 * tot_macs / (tot_ms * 1e-3) / 1e9}


def time_mbit(n, bits, reps=5, warmup=3, dev="cuda:0", seed=0):
    """Trigonometric encoder forward and backward on n elements (streaming kernels; GB/s of their algorithmic bytes)."""
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.rand(n, device=dev, generator=g) * 2 - 1
    c = torch.empty((bits, n), dtype=torch.float32, device=dev)
    gc = torch.randn((bits, n), device=dev, generator=g)
    gx = torch.empty(n, dtype=torch.float32, device=dev)
    tf = statistics.median(_time_calls(lambda i: qnn.mbit_encoder_forward(x, bits, 1.0, c=c), reps, warmup))
    tb = statistics.median(_time_calls(lambda i: qnn.mbit_encoder_backward(x, gc, bits, 1.0, gx=gx), reps, warmup))
    return {"call": "qnn_mbit_encoder", "n": n, "bits": bits, "forward_ms": tf, "backward_ms": tb,
            "forward_gbs": n * 4 * (1 + bits) / (tf * 1e-3) / 1e9, "backward_gbs": n * 4 * (2 + bits) / (tb * 1e-3) / 1e9}


def time_backward(m, n, k, ab, wb, reps=5, warmup=3, dev="cuda:0", seed=0):
    """Backward products of one FC layer (TF32 tensor-core contractions): whole calls, and the staging part alone."""
    g = torch.Generator(device=dev).manual_seed(seed)
    grad = torch.randn((m, n), device=dev, generator=g)
    x = (torch.rand((m, k), device=dev, generator=g) * 2 - 1)
    a_planes = qnn.encode_pack(x, ab, 1.0 / (2 ** ab - 1))
    w_planes = qnn.encode_pack(torch.randn((n, k), device=dev, generator=g).clamp_(-1, 1), wb, 1.0 / (2 ** wb - 1))
    alpha = 1.0 / ((2 ** ab - 1) * (2 ** wb - 1))
    out = torch.empty((m, k), dtype=torch.float32, device=dev)
    gw = torch.empty((n, k), dtype=torch.float32, device=dev)
    wsd = torch.empty(qnn.lib.qnn_bgemm_backward_data_workspace(m, n, k) + 256, dtype=torch.uint8, device=dev)
    wsw = torch.empty(qnn.lib.qnn_bgemm_backward_weights_workspace(m, n, k) + 256, dtype=torch.uint8, device=dev)
    med = lambda f: statistics.median(_time_calls(f, reps, warmup))
    td = med(lambda i: qnn.bgemm_backward_data(grad, w_planes, k, wb, alpha, out=out, workspace=wsd))
    te = med(lambda i: qnn.bgemm_backward_data(grad, w_planes, k, wb, alpha, x=x, ab=ab, r=1.0, out=out, workspace=wsd))
    tw = med(lambda i: qnn.bgemm_backward_weights(grad, a_planes, k, ab, alpha, gw=gw, workspace=wsw))
    tu = med(lambda i: qnn.unpack_codes_f32(w_planes, n, k, wb, transpose=True))
    status = qnn.tensor_path_status()
    fl = 2.0 * m * n * k
    return {"call": "qnn_bgemm_backward", "m": m, "n": n, "k": k, "ab": ab, "wb": wb, "status": status,
            "data_ms": td, "data_encoder_ms": te, "weights_ms": tw, "unpack_t_ms": tu,
            "data_tflops": fl / (td * 1e-3) / 1e12, "data_encoder_tflops": fl / (te * 1e-3) / 1e12,
            "weights_tflops": fl / (tw * 1e-3) / 1e12}


def time_backward_conv(N, H, W, C, Cout, R, S, stride, pad, ab, wb, reps=5, warmup=3, dev="cuda:0", seed=0):
    """Backward products of one convolution layer: whole calls (patch staging + TF32 tensor-core GEMM + gather)."""
    g = torch.Generator(device=dev).manual_seed(seed)
    Ho, Wo = qnn.conv_out_dim(H, R, stride, pad), qnn.conv_out_dim(W, S, stride, pad)
    grad = torch.randn((N, Ho, Wo, Cout), device=dev, generator=g)
    x = torch.rand((N * H * W, C), device=dev, generator=g) * 2 - 1
    a_planes = qnn.encode_pack(x, ab, 1.0 / (2 ** ab - 1))
    w = torch.randn((Cout, R, S, C), device=dev, generator=g).clamp_(-1, 1)
    packed = qnn.pack_weights(w, Cout, R * S, C, qnn.W_NTC, wb, 1.0 / (2 ** wb - 1))
    alpha = 1.0 / ((2 ** ab - 1) * (2 ** wb - 1))
    out = torch.empty((N, H, W, C), dtype=torch.float32, device=dev)
    gw = torch.empty((Cout, R, S, C), dtype=torch.float32, device=dev)
    wsd = torch.empty(qnn.lib.qnn_bconv2d_backward_data_workspace(N, H, W, C, Cout, R, S, stride, pad) + 256, dtype=torch.uint8, device=dev)
    wsw = torch.empty(qnn.lib.qnn_bconv2d_backward_weights_workspace(N, H, W, C, Cout, R, S, stride, pad) + 256, dtype=torch.uint8, device=dev)
    med = lambda f: statistics.median(_time_calls(f, reps, warmup))
    td = med(lambda i: qnn.bconv2d_backward_data(grad, packed, wb, H, W, C, R, S, stride, pad, alpha, out=out, workspace=wsd))
    tw = med(lambda i: qnn.bconv2d_backward_weights(grad, a_planes, ab, H, W, C, R, S, stride, pad, alpha, gw=gw, workspace=wsw))
    status = qnn.tensor_path_status()
    fl = 2.0 * N * Ho * Wo * Cout * R * S * C
    return {"call": "qnn_bconv2d_backward", "N": N, "H": H, "W": W, "C": C, "Cout": Cout, "R": R, "S": S, "stride": stride,
            "pad": pad, "ab": ab, "wb": wb, "status": status, "data_ms": td, "weights_ms": tw,
            "data_tflops": fl / (td * 1e-3) / 1e12, "weights_tflops": fl / (tw * 1e-3) / 1e12,
            "workspace_mb": [wsd.numel() / 1e6, wsw.numel() / 1e6]}


class ExpertsLayer:
    """A feed-forward layer of experts on 4-bit weights: every token goes through `top` of them, out = sum of gate * W2_e
    silu(W1_e x).  The real weights are kept for training: a step takes the gradient of the decoded weights for theirs
    (straight-through) and packs them again.  A 4-bit matrix reads the layer's output, as the last layer of a decoder would."""

    def __init__(self, hidden, inner, experts, top, classes, group=128, dtype=torch.bfloat16, seed=0, dev="cuda:0"):
        g = torch.Generator(device=dev).manual_seed(seed)
        self.top, self.group, self.dtype = top, group, dtype
        self.w1 = torch.randn((experts, inner, hidden), device=dev, generator=g) * hidden ** -0.5
        self.w2 = torch.randn((experts, hidden, inner), device=dev, generator=g) * inner ** -0.5
        self.router = torch.randn((experts, hidden), device=dev, generator=g) * hidden ** -0.5
        self.head = qnn.g4_pack_weights(torch.randn((classes, hidden), device=dev, generator=g) * hidden ** -0.5, group)
        self.pack()

    def pack(self):
        self.q1, self.q2 = qnn.g4_pack_weights(self.w1, self.group), qnn.g4_pack_weights(self.w2, self.group)

    def plan(self, x):
        """Rows sorted by expert: (token of each row, its gate, offsets); the split never leaves the device."""
        return self.route(x)[1:]

    def route(self, x):
        """The places that the sorted rows come from (token * top + choice), and plan's answer."""
        gate, expert = torch.softmax(x.float() @ self.router.t(), 1).topk(self.top, 1)
        flat = expert.reshape(-1)
        order = torch.sort(flat, stable=True).indices
        counts = (flat.view(-1, 1) == torch.arange(self.router.shape[0], device=x.device)).sum(0)
        offsets = torch.zeros(counts.numel() + 1, dtype=torch.int32, device=x.device)
        offsets[1:] = counts.cumsum(0)
        return order, order // self.top, (gate / gate.sum(1, keepdim=True)).reshape(-1)[order].to(x.dtype), offsets

    def forward(self, x):
        order, token, gate, offsets = self.route(x)
        rows = x[token]
        h = qnn.g4_expert_gemm(rows, self.q1, offsets)
        y = qnn.g4_expert_gemm(torch.nn.functional.silu(h), self.q2, offsets)
        slots = torch.empty_like(y)
        slots[order] = y * gate.view(-1, 1)                         # a token's rows together again, added in a fixed order
        out = slots.view(x.shape[0], self.top, -1).float().sum(1)
        return out.to(x.dtype), (token, gate, offsets, rows, h)

    def logits(self, x):
        return qnn.g4_matvec(self.forward(x)[0], self.head)

    def train_step(self, x, target, rate):
        """One step of gradient descent on 0.5 * mean squared error; the gates are held fixed.  Returns the loss."""
        out, (token, gate, offsets, rows, h) = self.forward(x)
        diff = out.float() - target
        dy = (diff[token] * gate.float().view(-1, 1)).to(x.dtype)
        a = torch.nn.functional.silu(h)
        dw2 = qnn.expert_gemm_backward_weights(dy, a, offsets)
        da = qnn.g4_expert_gemm_backward_data(dy, self.q2, offsets)
        s = torch.sigmoid(h.float())
        dh = (da.float() * s * (1 + h.float() * (1 - s))).to(x.dtype)
        dw1 = qnn.expert_gemm_backward_weights(dh, rows, offsets)
        dx = qnn.g4_expert_gemm_backward_data(dh, self.q1, offsets)          # what a layer below would be given
        self.w1 -= rate / x.shape[0] * dw1
        self.w2 -= rate / x.shape[0] * dw2
        self.pack()
        return float(0.5 * diff.square().sum(1).mean()), dx


def time_experts(tokens, experts, top, hidden, inner, group=128, dtype="bf16", reps=5, warmup=3, dev="cuda:0"):
    kind = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    layer = ExpertsLayer(hidden, inner, experts, top, 4 * hidden, group, kind, dev=dev)
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((tokens, hidden), device=dev, generator=g).to(kind)
    target = torch.randn((tokens, hidden), device=dev, generator=g)
    prompt = statistics.median(_time_calls(lambda i: layer.forward(x), reps, warmup))
    token = statistics.median(_time_calls(lambda i: layer.logits(x[:1]), reps, warmup))
    losses = []
    step = statistics.median(_time_calls(lambda i: losses.append(layer.train_step(x, target, 0.05)[0]), reps, warmup))
    return {"call": "experts", "tokens": tokens, "experts": experts, "top": top, "hidden": hidden, "inner": inner, "group": group,
            "dtype": dtype, "forward_ms": prompt, "one_token_ms": token, "train_step_ms": step, "first_loss": losses[0],
            "last_loss": losses[-1], "status": qnn.tensor_path_status()}


class FeedForwardBlock:
    """The feed-forward half of a decoder block: norm of x + residual, then a dense branch with weights and activations in 8 bits and,
    beside it, a layer of experts on 4-bit weights that sigmoid scores route to, balanced by a bias and limited to the best half of
    the groups:

        h = x + residual     y = rms_norm(h)     out = h + down(silu(up(y))) + sum of weight * W2_e silu(W1_e y)

    The real weights are kept for training: backward gives the gradients of the decoded ones, straight through every rounding."""

    def __init__(self, hidden, inner, experts, top, groups=1, group=64, dtype=torch.bfloat16, seed=0, dev="cuda:0"):
        g = torch.Generator(device=dev).manual_seed(seed)
        normal = lambda *shape: torch.randn(shape, device=dev, generator=g)
        self.top, self.groups, self.group, self.dtype, self.factor, self.eps = top, groups, group, dtype, 2.0, 1e-6
        self.gain = (1.0 + 0.1 * normal(hidden)).to(dtype)
        self.router, self.bias = normal(experts, hidden) * hidden ** -0.5, normal(experts) * 0.05
        self.w1, self.w2 = normal(experts, inner, hidden) * hidden ** -0.5, normal(experts, hidden, inner) * inner ** -0.5
        self.up, self.down = normal(2 * inner, hidden) * hidden ** -0.5, normal(hidden, 2 * inner) * (2 * inner) ** -0.5
        self.pack()

    def pack(self):
        self.q1, self.q2 = qnn.g4_pack_weights(self.w1, self.group), qnn.g4_pack_weights(self.w2, self.group)
        self.q_up, self.q_down = qnn.i8_quantize(self.up), qnn.i8_quantize(self.down)

    def forward(self, x, residual, mask=None):
        """x, residual [tokens, hidden]; mask (optional) [tokens], False for padding, which no expert sees.  Returns out and what
        backward needs."""
        silu = torch.nn.functional.silu
        rows, y, h, rstd = qnn.rms_norm_i8(x, self.gain, self.eps, residual, both=True)
        a = qnn.i8_gemm(rows, self.q_up, self.dtype)
        act = qnn.i8_quantize(silu(a))
        dense = qnn.i8_gemm(act, self.q_down, self.dtype)
        logits = y.float() @ self.router.t()
        routes = qnn.route(logits, self.top, "sigmoid", self.bias, self.groups, max(1, self.groups // 2), "top2", True, self.factor, mask)
        expert_rows = y[routes.order.clamp(min=0) // self.top]
        b = qnn.g4_expert_gemm(expert_rows, self.q1, routes.offsets)
        z = qnn.g4_expert_gemm(silu(b), self.q2, routes.offsets)
        there = (routes.place >= 0).unsqueeze(2)
        picked = torch.where(there, z[routes.place.clamp(min=0)].float(), 0.0)                # [tokens, top, hidden]
        out = h.float() + dense.float() + (picked * routes.weights.unsqueeze(2)).sum(1)
        return out.to(x.dtype), (rows, y, h, rstd, a, act, logits, routes, expert_rows, b, picked)

    def backward(self, dout, saved):
        """Gradients of sum(dout * out) with respect to x (the residual's too) and the weights."""
        rows, y, h, rstd, a, act, logits, routes, expert_rows, b, picked = saved
        everything = torch.tensor([0, y.shape[0]], dtype=torch.int32, device=y.device)
        dsilu = lambda v: (lambda s: s * (1 + v.float() * (1 - s)))(torch.sigmoid(v.float()))
        d = dout.to(self.dtype)
        grads = {"down": qnn.expert_gemm_backward_weights(d, qnn.i8_decode(act, self.dtype), everything)[0]}
        da = ((d.float() @ qnn.i8_decode(self.q_down, torch.float32)) * dsilu(a)).to(self.dtype)
        grads["up"] = qnn.expert_gemm_backward_weights(da, qnn.i8_decode(rows, self.dtype), everything)[0]
        dy = da.float() @ qnn.i8_decode(self.q_up, torch.float32)
        slot = routes.order.clamp(min=0)
        dz = (d.float()[slot // self.top] * routes.weights.reshape(-1)[slot].unsqueeze(1)).to(self.dtype)
        grads["w2"] = qnn.expert_gemm_backward_weights(dz, torch.nn.functional.silu(b), routes.offsets)
        db = (qnn.g4_expert_gemm_backward_data(dz, self.q2, routes.offsets).float() * dsilu(b)).to(self.dtype)
        grads["w1"] = qnn.expert_gemm_backward_weights(db, expert_rows, routes.offsets)
        drows = qnn.g4_expert_gemm_backward_data(db, self.q1, routes.offsets)
        dy += torch.where((routes.place >= 0).unsqueeze(2), drows[routes.place.clamp(min=0)].float(), 0.0).sum(1)
        dlogits = qnn.route_backward((picked * d.float().unsqueeze(1)).sum(2), logits, routes.experts, "sigmoid", True, self.factor)
        grads["router"] = dlogits.t() @ y.float()
        dy += dlogits @ self.router
        grads["x"], grads["gain"] = qnn.rms_norm_backward(dy.to(self.dtype), h, self.gain, rstd, d)
        return grads

    def train_step(self, x, residual, target, rate):
        """One step of gradient descent on 0.5 * mean squared error.  Returns the loss."""
        out, saved = self.forward(x, residual)
        diff = out.float() - target
        grads = self.backward(diff / x.shape[0], saved)
        for name in ("w1", "w2", "up", "down", "router"):
            getattr(self, name).sub_(rate * grads[name])
        self.gain = (self.gain.float() - rate * grads["gain"]).to(self.dtype)
        self.pack()
        return float(0.5 * diff.square().sum(1).mean())


def time_block(tokens, experts, top, groups, hidden, inner, dtype="bf16", reps=5, warmup=3, dev="cuda:0"):
    kind = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    block = FeedForwardBlock(hidden, inner, experts, top, groups, dtype=kind, dev=dev)
    g = torch.Generator(device=dev).manual_seed(1)
    x, residual = (torch.randn((tokens, hidden), device=dev, generator=g).to(kind) for _ in range(2))
    target = torch.randn((tokens, hidden), device=dev, generator=g)
    prompt = statistics.median(_time_calls(lambda i: block.forward(x, residual), reps, warmup))
    token = statistics.median(_time_calls(lambda i: block.forward(x[:1], residual[:1]), reps, warmup))
    losses = []
    step = statistics.median(_time_calls(lambda i: losses.append(block.train_step(x, residual, target, 0.05)), reps, warmup))
    return {"call": "block", "tokens": tokens, "experts": experts, "top": top, "groups": groups, "hidden": hidden, "inner": inner,
            "dtype": dtype, "forward_ms": prompt, "one_token_ms": token, "train_step_ms": step, "first_loss": losses[0],
            "last_loss": losses[-1], "status": qnn.tensor_path_status()}


def _report(call, Mg, Ng, Kg, ab, wb, times):
    ms = statistics.median(times)
    macs = float(Mg) * Ng * Kg
    return {"call": call, "Mg": Mg, "Ng": Ng, "Kg": Kg, "ab": ab, "wb": wb, "ms_median": ms, "ms_min": min(times),
            "binary_tops": 2 * macs * ab * wb / (ms * 1e-3) / 1e12, "equiv_int_gops": 2 * macs / (ms * 1e-3) / 1e9,
            "bytes": Mg * Kg * ab / 8 + Ng * Kg * wb / 8 + Mg * Ng * 4}


def main():
    ap = argparse.ArgumentParser()
    sub = ap.add_subparsers(dest="case", required=True)
    g = sub.add_parser("gemm")
    for name, default in (("m", 4096), ("n", 4096), ("k", 4096), ("ab", 2), ("wb", 2)):
        g.add_argument(f"--{name}", type=int, default=default)
    c = sub.add_parser("conv")
    for name, default in (("N", 32), ("H", 14), ("W", 14), ("C", 256), ("Cout", 256), ("R", 3), ("S", 3),
                          ("stride", 1), ("pad", 1), ("ab", 2), ("wb", 2)):
        c.add_argument(f"--{name}", type=int, default=default)
    e = sub.add_parser("encode")
    for name, default in (("rows", 4096), ("k", 4096), ("bits", 2)):
        e.add_argument(f"--{name}", type=int, default=default)
    mb = sub.add_parser("mbit")
    mb.add_argument("--n", type=int, default=1 << 26)
    mb.add_argument("--bits", type=int, default=2)
    bw = sub.add_parser("backward")
    bw.add_argument("--m", type=int, default=4096)
    bw.add_argument("--n", type=int, default=4096)
    bw.add_argument("--k", type=int, default=4096)
    bw.add_argument("--ab", type=int, default=2)
    bw.add_argument("--wb", type=int, default=2)
    bc = sub.add_parser("backward_conv")
    for name, default in (("N", 32), ("H", 14), ("W", 14), ("C", 256), ("Cout", 256), ("R", 3), ("S", 3),
                          ("stride", 1), ("pad", 1), ("ab", 2), ("wb", 2)):
        bc.add_argument(f"--{name}", type=int, default=default)
    k = sub.add_parser("stack")
    k.add_argument("--net", choices=["resnet18", "resnet18_p1", "resnet18_p2", "vgg16"], default="resnet18")
    k.add_argument("--batch", type=int, default=0)
    k.add_argument("--layers", type=str, default="")
    k.add_argument("--table", action="store_true")
    x = sub.add_parser("experts")
    for name, default in (("tokens", 512), ("experts", 8), ("top", 2), ("hidden", 1024), ("inner", 2048), ("group", 128)):
        x.add_argument(f"--{name}", type=int, default=default)
    x.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    fb = sub.add_parser("block")
    for name, default in (("tokens", 512), ("experts", 32), ("top", 4), ("groups", 4), ("hidden", 1024), ("inner", 512)):
        fb.add_argument(f"--{name}", type=int, default=default)
    fb.add_argument("--dtype", choices=["bf16", "fp16", "fp32"], default="bf16")
    for s in (g, c, e, k, mb, bw, bc, x, fb):
        s.add_argument("--reps", type=int, default=5)
        s.add_argument("--warmup", type=int, default=3)
        s.add_argument("--sets", type=int, default=3)
    a = ap.parse_args()
    if a.case == "gemm":
        r = time_gemm(a.m, a.n, a.k, a.ab, a.wb, a.reps, a.warmup, a.sets)
    elif a.case == "conv":
        r = time_conv(a.N, a.H, a.W, a.C, a.Cout, a.R, a.S, a.stride, a.pad, a.ab, a.wb, a.reps, a.warmup, a.sets)
    elif a.case == "backward":
        r = time_backward(a.m, a.n, a.k, a.ab, a.wb, a.reps, a.warmup)
    elif a.case == "backward_conv":
        r = time_backward_conv(a.N, a.H, a.W, a.C, a.Cout, a.R, a.S, a.stride, a.pad, a.ab, a.wb, a.reps, a.warmup)
    elif a.case == "experts":
        r = time_experts(a.tokens, a.experts, a.top, a.hidden, a.inner, a.group, a.dtype, a.reps, a.warmup)
    elif a.case == "block":
        r = time_block(a.tokens, a.experts, a.top, a.groups, a.hidden, a.inner, a.dtype, a.reps, a.warmup)
    elif a.case == "mbit":
        r = time_mbit(a.n, a.bits, a.reps, a.warmup)
    elif a.case == "stack":
        batch = a.batch or (64 if a.net == "vgg16" else 256)
        layers = [int(v) for v in a.layers.split(",")] if a.layers else None
        r = time_stack(a.net, batch, a.reps, a.warmup, layers=layers)
        if a.table:
            print(f"{'layer':28s} {'Mg':>8s} {'Ng':>4s} {'Kg':>5s} {'enc ms':>8s} {'conv ms':>8s} {'bTOPS':>7s} {'enc GB/s':>8s} {'conv+enc fused ms':>18s}")
            for L in r["layers"]:
                print(f"{L['layer']:28s} {L['Mg']:8d} {L['Ng']:4d} {L['Kg']:5d} {L['encode_ms']:8.3f} {L['conv_ms']:8.3f} "
                      f"{L['conv_binary_tops']:7.1f} {L['encode_gbs']:8.0f} {L['conv_encode_ms']:18.3f}")
            print(f"total {r['total_ms']:.3f} ms (encode + conv per layer), {r['binary_tops']:.1f} binary TOPS, "
                  f"{r['equiv_int_gops']:.0f} equiv int GOPS; chained plane-to-plane (fused encoder, no fp32 between "
                  f"layers): {sum(L['conv_encode_ms'] for L in r['layers']):.3f} ms")
            return
    else:
        r = time_encode(a.rows, a.k, a.bits, a.reps, a.warmup, a.sets)
    print(json.dumps(r))


if __name__ == "__main__":
    main()

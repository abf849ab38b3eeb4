#!/usr/bin/env python3
"""The backbone of a decoder layer in 8-bit integers, next to its LoRA add-ons, as cases that can be timed and compared.

The add-ons land on the outputs of dense projections.  Where the model's own weights are held in 8 bits, a layer
runs, on the token rows of one batch:

  norm       rms norm of (x + residual): the sum, the normed rows in 16 bits (what the add-ons read) and in 8 bits
             with a scale per row (what the projections read)
  dense      y = (q W^T) * row scale * channel scale for one to three projections of the same rows, q and W in 8 bits
  silu       silu(gate) * up, in 16 bits and in 8 bits with a scale per row (between gate / up and down, after
             their add-ons)
  quantize   16-bit rows in 8 bits with a scale per row (the attention's output in front of the o projection)

Fields of a case
  op         one of the four
  dtype      "f16" or "bf16": type of everything that is not 8-bit or a scale
  rows       token rows of the batch
  h          width of the rows; for "dense" that of its input
  outs       "dense": output widths of the projections, "4096,1024,1024"
  residual   "norm": whether there is a residual to add
  out16      "norm" and "silu": whether the rows are wanted in 16 bits too

8-bit rows are returned as the values they stand for, q * scale, in the case's 16-bit type.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
SCRATCH = 16 << 20  # bytes of scratch memory that a program keeps for its dense projections
_DEFAULTS = dict(op="dense", dtype="f16", rows=1, h=4096, outs="", residual=False, out16=False)


def _case(**fields):
    return {**_DEFAULTS, **fields}


def listed():
    return [
        # one user's decode row on its way into q / k / v: the smallest call, launch and host cost
        _case(name="norm_1", op="norm", residual=True, out16=True),
        # an odd batch through a layer of an odd width, without a residual (the first layer of a model)
        _case(name="norm_577_odd", op="norm", dtype="bf16", rows=577, h=5128, out16=True),
        # prompts of eight requests on a wide model
        _case(name="norm_prefill_bf16", op="norm", dtype="bf16", rows=4814, h=8192, residual=True, out16=True),
        # a decode batch in front of the MLP's down projection
        _case(name="silu_64", op="silu", rows=64, h=11008, out16=True),
        # prompts in front of the down projection of a 13B-sized model
        _case(name="silu_prefill_bf16", op="silu", dtype="bf16", rows=2900, h=13824, out16=True),
        # a decode batch's attention output
        _case(name="quantize_45_bf16", op="quantize", dtype="bf16", rows=45, h=5120),
        # prompts' attention output
        _case(name="quantize_prefill", op="quantize", rows=8190, h=4096),
        # one decode row, q / k / v: all of the three weights from memory
        _case(name="dense_1_qkv", rows=1, outs="4096,4096,4096"),
        # the headline decode batch, gate / up
        _case(name="dense_64_gate_up", rows=64, outs="11008,11008"),
        # an odd decode batch, the widest input of a 13B-sized model
        _case(name="dense_45_down_bf16", dtype="bf16", rows=45, h=13824, outs="5120"),
        # decode rows next to a prompt, q / k / v with shared heads
        _case(name="dense_mixed_517_qkv", rows=517, outs="4096,1024,1024"),
        # prompts of eight requests, MLP-sized output: the largest matrix product
        _case(name="dense_prefill_mlp_bf16", dtype="bf16", rows=4814, h=8192, outs="28672"),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng):
    """Usual widths, and every other one: a multiple of 8 in [256, 13824]."""
    if rng.random() < 0.5:
        return rng.choice((1024, 2048, 4096, 5120, 8192, 11008, 13824))
    return max(256, _log_uniform(rng, 256, 13824) // 8 * 8)


def draw(rng):
    op = rng.choice(("norm", "silu", "quantize", "dense", "dense", "dense"))
    c = _case(op=op, dtype=rng.choice(("f16", "bf16")), h=_width(rng))
    if op == "dense":
        outs = [_width(rng) for _ in range(rng.randint(1, 3))]
        c["outs"] = ",".join(map(str, outs))
        c["rows"] = _log_uniform(rng, 1, min(8192, 2.2e12 / (2 * c["h"] * sum(outs))))
    else:
        c["rows"] = _log_uniform(rng, 1, min(16384, 3.9e7 / c["h"]))
        c["out16"] = op != "quantize" and rng.random() < 0.8
        c["residual"] = op == "norm" and rng.random() < 0.8
    return c


def _outs(case):
    return [int(n) for n in case["outs"].split(",")] if case["outs"] else []


def work(case):
    m, h = case["rows"], case["h"]
    if case["op"] == "dense":
        n = sum(_outs(case))
        return {"bytes": m * h + 4 * m + n * (h + 4) + 2 * m * n, "flops": 2 * m * n * h}
    read = {"norm": 4 if case["residual"] else 2, "silu": 4, "quantize": 2}[case["op"]]
    written = 1 + 2 * case["out16"] + 2 * case["residual"]
    return {"bytes": m * h * (read + written) + 4 * m + (2 * h if case["op"] == "norm" else 0),
            "flops": m * h * {"norm": 8, "silu": 10, "quantize": 3}[case["op"]]}


def _activations(gen, rows, h, dtype):
    """Activations of a language model: normal, with a few channels that are much larger in every row."""
    wide = 1.0 + 19.0 * (torch.rand(h, generator=gen, device="cuda") < 0.003)
    return (torch.randn(rows, h, generator=gen, device="cuda") * wide).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    m, h, t, op = case["rows"], case["h"], TORCH[case["dtype"]], case["op"]

    def new(*shape, dtype=t):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s = {"case": case, "op": op, "q": new(m, h, dtype=torch.int8), "scales": new(m, dtype=torch.float32)}
    if op == "dense":
        x = _activations(gen, m, h, torch.float32)
        top = x.abs().amax(1, keepdim=True)
        s["q"] = (x * (127.0 / top)).round_().to(torch.int8)
        s["scales"] = (top[:, 0] / 127.0).contiguous()
        s["outs"] = _outs(case)
        s["scratch"] = new(SCRATCH, dtype=torch.uint8)
        s["w"], s["w_scales"], s["y"] = [], [], []
        for n in s["outs"]:
            # weights as a per-channel quantiser leaves them: the largest of a channel's normal values is 127
            s["w"].append((torch.randn(n, h, generator=gen, device="cuda") * 32.0).round_().clamp_(-127, 127).to(torch.int8))
            s["w_scales"].append((0.5 + torch.rand(n, generator=gen, device="cuda")) / (32.0 * math.sqrt(h)))
            s["y"].append(new(m, n))
        return s
    s["x"] = _activations(gen, m, h, t)
    s["values"] = new(m, h)
    s["out"] = new(m, h) if case["out16"] else None
    if op == "norm":
        s["weight"] = (1.0 + 0.2 * torch.randn(h, generator=gen, device="cuda")).to(t)
        s["residual"] = _activations(gen, m, h, t) if case["residual"] else None
        s["sum"] = new(m, h) if case["residual"] else None
    if op == "silu":
        s["up"] = _activations(gen, m, h, t)
    return s


def _quantized(v):
    """Scale of each row and the values that its 8-bit integers stand for."""
    top = v.abs().amax(1, keepdim=True)
    scales = top / 127.0
    q = torch.where(top > 0, torch.round(v * (127.0 / top)), torch.zeros_like(v))
    return scales, q * scales


def _plain(s):
    t = TORCH[s["case"]["dtype"]]
    if s["op"] == "dense":
        x, sx = s["q"].float(), s["scales"][:, None]
        return [((x @ w.float().t()) * sx * sw).to(t) for w, sw in zip(s["w"], s["w_scales"])]
    v, total = s["x"].float(), None
    if s["op"] == "norm":
        if s["residual"] is not None:
            v = v + s["residual"].float()
            total = v.to(t)
        v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["weight"].float()
    elif s["op"] == "silu":
        v = v / (1.0 + torch.exp(-v)) * s["up"].float()
    scales, values = _quantized(v)
    return {"scales": scales[:, 0], "values": values.to(t), "out": v.to(t) if s["out"] is not None else None, "sum": total}


def _calls(s):
    from paper_2310_18547_amd import binding as B
    case, op = s["case"], s["op"]
    m, h, t = case["rows"], case["h"], B.F16 if case["dtype"] == "f16" else B.BF16
    stream = torch.cuda.current_stream().cuda_stream
    if op == "dense":
        B.sgmv_dense_q8(t, s["y"], s["q"], s["scales"], s["w"], s["w_scales"], m, h, s["outs"], s["scratch"], SCRATCH, stream)
        return s["y"]
    if op == "norm":
        B.sgmv_rms_norm_q8(t, s["out"], s["q"], s["scales"], s["sum"], s["x"], s["residual"], s["weight"], EPS, m, h, stream)
    elif op == "silu":
        B.sgmv_silu_mul_q8(t, s["out"], s["q"], s["scales"], s["x"], s["up"], m, h, stream)
    else:
        B.sgmv_quantize_q8(t, s["q"], s["scales"], s["x"], m, h, stream)
    torch.mul(s["q"], s["scales"][:, None], out=s["values"])
    return {"scales": s["scales"], "values": s["values"], "out": s["out"], "sum": s.get("sum")}


def run(state):
    return _calls(state) if own else _plain(state)


def exact(case, seed):
    s = prepare(case, seed)
    m, h = case["rows"], case["h"]
    if case["op"] == "dense":
        q = s["q"].to(torch.float64)
        # whole numbers below 2^53 all along: the sums are exact in 64 bits
        return [torch.matmul(q, w.to(torch.float64).t()).mul_(sw.to(torch.float64)).mul_(s["scales"].to(torch.float64).view(m, 1))
                for w, sw in zip(s["w"], s["w_scales"])]
    result = {"scales": None, "values": None, "out": None, "sum": None}
    rows = s["x"].to(torch.float64)
    if case["op"] == "norm":
        if case["residual"]:
            rows += s["residual"].to(torch.float64)
            result["sum"] = rows.clone()
        power = torch.linalg.vector_norm(rows, dim=1).square() / h
        rows = rows / torch.sqrt(power + EPS).view(m, 1) * s["weight"].to(torch.float64)
    elif case["op"] == "silu":
        rows = rows * torch.sigmoid(rows) * s["up"].to(torch.float64)
    if case["out16"]:
        result["out"] = rows
    step = torch.linalg.vector_norm(rows, ord=math.inf, dim=1) / 127.0
    result["scales"] = step
    result["values"] = torch.round(rows / step.clamp_min(np.finfo(np.float64).tiny).view(m, 1)) * step.view(m, 1)
    return result

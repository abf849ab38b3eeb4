"""A decoder layer on the 8-bit backbone: norms, projections with their add-ons and the gated activation together, as a program
runs them, every stage against its definition in 64 bits from what the stage before it left."""
import numpy as np
import pytest
import torch

import backbone_reference as ref
import sgmv_workloads as wl
from helpers import decode64, tolerance

pytestmark = pytest.mark.gpu
KIND = {"f16": torch.float16, "bf16": torch.bfloat16}


def _host(t):
    a = t.cpu().view(torch.int16) if t.dtype in (torch.float16, torch.bfloat16) else t.cpu()
    a = a.numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


class _Layer:
    """Weights, adapters and a Q8Layer for segments of the given lengths (every segment an adapter of its own)."""

    def __init__(self, lens, dtype, h=520, ffn=1384, r=16, layers=2, seed=0):
        from paper_2310_18547_amd import binding as B
        from paper_2310_18547_amd.device import DeviceWorkload
        from paper_2310_18547_amd.layer import Q8Layer, projection_shapes, quantize_weight
        self.dtype, self.n, self.lens = dtype, sum(lens), lens
        shapes = projection_shapes(h, ffn)
        self.loads = {name: wl.custom(lens, i, o, r, dtype, num_layers=layers, seed=seed + k)
                      for k, (name, (i, o)) in enumerate(shapes.items())}
        self.d = {name: DeviceWorkload(w, "cuda:0", init_workspace=False) for name, w in self.loads.items()}
        gen = torch.Generator(device="cuda:0").manual_seed(seed)
        self.weights = {name: [quantize_weight(torch.randn(o, i, generator=gen, device="cuda:0") * i ** -0.5) for _ in range(layers)]
                        for name, (i, o) in shapes.items()}
        norms = [tuple((1 + 0.2 * torch.randn(h, generator=gen, device="cuda:0")).to(KIND[dtype]) for _ in range(2)) for _ in range(layers)]
        self.layer = Q8Layer(h, ffn, r, layers, self.n, B.F16 if dtype == "f16" else B.BF16,
                             {k: d.A_ptrs for k, d in self.d.items()}, {k: d.B_ptrs for k, d in self.d.items()},
                             self.d["q"].seg_starts, len(lens), max(lens), self.weights, norms)
        self.norms = norms
        self.rows = lambda: torch.randn(self.n, h, generator=gen, device="cuda:0").to(KIND[dtype])

    def add_on(self, name, x, layer_idx):
        """x A B of every row, in 64 bits."""
        w, x = self.loads[name], decode64(x, self.dtype)
        out, lo = np.zeros((self.n, w.h_out)), 0
        for i, length in enumerate(self.lens):
            a, b = decode64(w.A[i][layer_idx], self.dtype), decode64(w.B[i][layer_idx], self.dtype)
            out[lo:lo + length] = x[lo:lo + length] @ a @ b
            lo += length
        return out

    def check_projection(self, name, q, scales, x, layer_idx, scale):
        w, s = self.weights[name][layer_idx]
        backbone = decode64(ref.dense(_host(q), _host(scales), _host(w), _host(s), self.dtype), self.dtype)
        want = backbone + scale * self.add_on(name, _host(x), layer_idx)
        got = decode64(_host(self.layer.y[name]), self.dtype)
        assert np.all(np.abs(got - want) <= tolerance(want)), name
        assert np.abs(want - backbone).max() > 0.1, "the add-on is there"

    def check_norm(self, which, x, residual_before, residual_after, layer_idx):
        L = self.layer
        w = _host(self.norms[layer_idx][which])
        s, v = ref.norm(residual_before, x, w, np.float32(L.eps), self.dtype)
        ref.check_rows(v, _host(L.x), _host(L.q), _host(L.q_scales).astype(np.float64), self.dtype, "norm")
        off = np.abs(decode64(residual_after, self.dtype) - s)
        assert np.all(off <= np.abs(s) * (ref.HALF_STEP[self.dtype] + 2.0 ** -23) + ref.SMALLEST[self.dtype])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens", [[1] * 12, [1], [40, 1, 1, 0, 33, 1, 60]])
def test_layer_stage_by_stage(lens, dtype):
    t = _Layer(lens, dtype)
    L, scale = t.layer, 0.5
    residual, x = t.rows(), t.rows()
    for layer_idx in (0, 1):
        before = _host(residual).copy()
        L.qkv(x, residual, layer_idx, scale)
        t.check_norm(0, _host(x), before, _host(residual), layer_idx)
        for name in ("q", "k", "v"):
            t.check_projection(name, L.q, L.q_scales, L.x, layer_idx, scale)
        attention = L.y["v"].clone()
        # finish(), stage by stage
        from paper_2310_18547_amd import binding as B
        B.sgmv_quantize_q8(L.dtype, L.q, L.q_scales, attention, t.n, L.h)
        ref.check_rows(decode64(_host(attention), dtype), None, _host(L.q), _host(L.q_scales).astype(np.float64), dtype, "quantize")
        L.project(("o",), L.q, attention, layer_idx, scale)
        t.check_projection("o", L.q, L.q_scales, attention, layer_idx, scale)
        o, before = _host(L.y["o"]).copy(), _host(residual).copy()
        again = residual.clone()
        L.norm(1, L.y["o"], residual, layer_idx)
        t.check_norm(1, o, before, _host(residual), layer_idx)
        L.project(("gate", "up"), L.q, L.x, layer_idx, scale)
        for name in ("gate", "up"):
            t.check_projection(name, L.q, L.q_scales, L.x, layer_idx, scale)
        g, u = _host(L.y["gate"]), _host(L.y["up"])
        B.sgmv_silu_mul_q8(L.dtype, L.act, L.q_ffn, L.q_scales, L.y["gate"], L.y["up"], t.n, L.ffn)
        v = ref.silu_mul(g, u, dtype)
        ref.check_rows(v, _host(L.act), _host(L.q_ffn), _host(L.q_scales).astype(np.float64), dtype, "silu", ref.silu_extra(g, u, v, dtype))
        L.project(("down",), L.q_ffn, L.act, layer_idx, scale)
        t.check_projection("down", L.q_ffn, L.q_scales, L.act, layer_idx, scale)
        down = L.y["down"].clone()
        # the same in one call
        assert torch.equal(L.finish(attention, again, layer_idx, scale), down) and torch.equal(again, residual)
        x = down
    assert L.check() == 0


def test_layer_captured_and_replayed():
    """Two layers in a HIP graph: replays with new inputs give what eager calls give, the eager work in between."""
    t = _Layer([1, 3, 1, 2, 1], "f16", seed=4)
    L = t.layer
    x, residual = t.rows(), t.rows()
    static_x, static_residual = x.clone(), residual.clone()
    stream = torch.cuda.Stream(device="cuda:0")

    def step(x, residual, stream):
        for layer_idx in (0, 1):
            L.qkv(x if layer_idx == 0 else L.y["down"], residual, layer_idx, stream=stream)
            L.finish(L.y["v"], residual, layer_idx, stream=stream)
        return L.y["down"]

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(static_x, static_residual, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(static_x, static_residual, torch.cuda.current_stream())
    for _ in range(4):
        x, residual = t.rows(), t.rows()
        static_x.copy_(x)
        static_residual.copy_(residual)
        torch.cuda.synchronize()
        want = step(x, residual, None).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.y["down"], want) and torch.equal(static_residual, residual)
    assert L.check() == 0


def test_layer_without_add_ons_and_first_layer():
    t = _Layer([2, 5], "bf16", seed=8)
    L = t.layer
    residual = t.rows()
    before = residual.clone()
    L.add_ons = False
    L.qkv(None, residual, 1)
    assert torch.equal(residual, before)            # nothing to add: the residual is left as it is
    for name in ("q", "k", "v"):
        w, s = t.weights[name][1]
        same = np.array_equal(_host(L.y[name]), ref.dense(_host(L.q), _host(L.q_scales), _host(w), _host(s), "bf16"))
        assert same, name

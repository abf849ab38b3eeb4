"""The seven LoRA add-ons of one decoder layer (call plumbing only).

The paper applies LoRA to every dense projection of a transformer layer -- query, key,
value, output, gate, up, down -- and builds the segment indices once per model invocation,
so one ``seg_starts`` serves all of them (Background, "Low-Rank Adaptation"; the remark on
segment indices in the section on the runner).  ``LoraLayer`` issues those seven add-ons
through the C ABI: the projections that read the same activations (q/k/v, gate/up) go into
one ``sgmv_add_lora_multi`` call each, o and down are single ``sgmv_add_lora`` calls.  All
calls share one workspace and must be enqueued on one stream.

``Q8Layer`` is a layer whose own weights are held in 8-bit integers: besides the add-ons it
issues the norms, the dense projections and the gated activation that they stand between,
everything of the layer but attention.
"""
from __future__ import annotations

from typing import Dict, Sequence

import torch

from . import binding as B

PROJECTIONS = ("q", "k", "v", "o", "gate", "up", "down")
GROUPS = (("q", "k", "v"), ("o",), ("gate", "up"), ("down",))


def projection_shapes(h: int, ffn: int) -> Dict[str, tuple]:
    """name -> (h_in, h_out) of a Llama-style decoder layer."""
    return {"q": (h, h), "k": (h, h), "v": (h, h), "o": (h, h), "gate": (h, ffn), "up": (h, ffn),
            "down": (ffn, h)}


class LoraLayer:
    def __init__(self, h: int, ffn: int, r: int, num_layers: int, n_tokens: int, dtype: int,
                 A_ptrs: Dict[str, torch.Tensor], B_ptrs: Dict[str, torch.Tensor],
                 seg_starts: torch.Tensor, n_segs: int, max_seg_len: int, device="cuda:0"):
        self.shapes = projection_shapes(h, ffn)
        self.A_ptrs, self.B_ptrs = A_ptrs, B_ptrs
        self.seg_starts, self.n_segs = seg_starts, n_segs
        self.ws_bytes = max(B.sgmv_workspace_bytes_multi(n_tokens, r, max(len(g) for g in GROUPS)), 256)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        B.sgmv_workspace_init(self.workspace, self.ws_bytes)
        torch.cuda.synchronize(device)
        self.problem = {n: B.make_problem(dtype, i, o, r, num_layers, n_tokens,
                                          workspace=self.workspace, workspace_bytes=self.ws_bytes,
                                          max_seg_len=max_seg_len, workspace_ready=1)
                        for n, (i, o) in self.shapes.items()}

    def add_lora(self, name: str, y, x, layer_idx: int, scale: float = 1.0, stream=None):
        return B.sgmv_add_lora(self.problem[name], y, x, self.A_ptrs[name], self.B_ptrs[name],
                               self.seg_starts, self.n_segs, layer_idx, scale, stream)

    def add_lora_group(self, names: Sequence[str], ys, xs, layer_idx: int, scale: float = 1.0,
                       stream=None):
        """Projections of one shape in one call (``ys`` / ``xs`` in the order of ``names``)."""
        if len(names) == 1:
            return self.add_lora(names[0], ys[0], xs[0], layer_idx, scale, stream)
        return B.sgmv_add_lora_multi(self.problem[names[0]], list(ys), list(xs),
                                     [self.A_ptrs[n] for n in names],
                                     [self.B_ptrs[n] for n in names], self.seg_starts,
                                     self.n_segs, layer_idx, scale, stream)

    def check(self, stream=None) -> int:
        return B.sgmv_workspace_check(self.workspace, stream)


def quantize_weight(w: torch.Tensor):
    """A projection's weight ``[h_out, h_in]`` in 8-bit integers with a scale per output channel (once, at loading).
    Weights that are not finite raise ``ValueError``."""
    scales = w.float().abs().amax(1, keepdim=True) / 127.0
    if not torch.isfinite(scales).all():
        raise ValueError("weights that are not finite have no 8-bit form")
    scales = torch.where(scales > 0, scales, torch.ones_like(scales))
    # the smallest scales have few bits: a quotient may pass 127
    return torch.round(w.float() / scales).clamp(-127, 127).to(torch.int8).contiguous(), scales[:, 0].contiguous()


def _require(t, kind, rows: int, width: int, device, what: str, exactly: bool = False) -> None:
    """Raises ``ValueError`` unless ``t`` holds ``rows`` rows or more of ``width`` values (one or several last dimensions together)
    without gaps; ``exactly``: is ``[rows, width]`` itself.  Its address is all that a call gets: anything else would be read as
    something else, or past its end.  An ``int`` is an address that the caller answers for."""
    if isinstance(t, int) and not exactly:
        return
    got = f"{type(t)!r}"
    if isinstance(t, torch.Tensor):
        values = 1
        for n in reversed(t.shape):
            values *= n
            if values >= width:
                break
        fits = tuple(t.shape) == (rows, width) if exactly else values == width and t.numel() >= rows * width
        if fits and t.dtype == kind and t.device == device and t.is_contiguous():
            return
        got = f"{tuple(t.shape)} of {t.dtype} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}"
    raise ValueError(f"{what}: {rows} contiguous rows of {width} {kind} on {device}, not {got}")


class Q8Layer(LoraLayer):
    """A decoder layer with an 8-bit backbone and 16-bit LoRA add-ons, for batches of ``n_tokens`` rows.

    ``weights`` holds, for every name of ``PROJECTIONS``, a list with a layer's ``(int8 [h_out, h_in], fp32 [h_out])`` for every
    layer; ``norms`` the 16-bit norm weights of every layer, ``(in front of attention, in front of the MLP)``.  Tensors
    of another type, shape, layout or device raise ``ValueError``, and so do rows in a buffer of the object that the call writes
    before it last reads them.  The buffers are the object's own and are used again by the next call: one call at a time, on one
    stream.
    """

    def __init__(self, h: int, ffn: int, r: int, num_layers: int, n_tokens: int, dtype: int, A_ptrs, B_ptrs, seg_starts,
                 n_segs: int, max_seg_len: int, weights, norms, eps: float = 1e-5, device="cuda:0"):
        super().__init__(h, ffn, r, num_layers, n_tokens, dtype, A_ptrs, B_ptrs, seg_starts, n_segs, max_seg_len, device)
        self.dtype, self.n_tokens, self.h, self.ffn, self.eps = dtype, n_tokens, h, ffn, eps
        self.weights, self.norms = weights, norms
        self.add_ons = True  # False: the backbone alone (benchmarks compare the two)
        self.kind = kind = torch.float16 if dtype == B.F16 else torch.bfloat16
        on = self.workspace.device
        for name, (h_in, h_out) in self.shapes.items():
            if len(weights[name]) < num_layers:
                raise ValueError(f"{name}: weights of {len(weights[name])} layers, not {num_layers}")
            for w, s in weights[name]:
                _require(w, torch.int8, h_out, h_in, on, f"weight of {name}", exactly=True)
                _require(s[None], torch.float32, 1, h_out, on, f"weight scales of {name}", exactly=True)
        if len(norms) < num_layers:
            raise ValueError(f"norm weights of {len(norms)} layers, not {num_layers}")
        for pair in norms:
            for w in pair:
                _require(w, kind, 1, h, on, "norm weight")

        def rows(width, kind=kind):
            return torch.empty(n_tokens, width, dtype=kind, device=device)

        self.y = {name: rows(h_out) for name, (_, h_out) in self.shapes.items()}
        self.x, self.act = rows(h), rows(ffn)                            # normed rows, gated activations
        self.q, self.q_ffn = rows(h, torch.int8), rows(ffn, torch.int8)  # in 8 bits
        self.q_scales = torch.empty(n_tokens, dtype=torch.float32, device=device)
        self.scratch = torch.empty(B.DENSE_WORKSPACE_BYTES, dtype=torch.uint8, device=device)
        self._own = {id(t): (t, t.shape[1], t.dtype) for t in (*self.y.values(), self.x, self.act, self.q, self.q_ffn)}

    def _rows(self, t, width: int, what: str, kind=None) -> None:
        """Checks a caller's rows; the object's own buffers are known."""
        kind = kind or self.kind
        own = self._own.get(id(t))
        if own is None or own[1:] != (width, kind):
            _require(t, kind, self.n_tokens, width, self.x.device, what)

    def _apart(self, t, buffers, what: str) -> None:
        """Refuses a tensor in one of the object's own buffers that the call writes before it last reads the tensor."""
        if isinstance(t, torch.Tensor) and t.numel() and t.untyped_storage().data_ptr() in [b.untyped_storage().data_ptr() for b in buffers]:
            raise ValueError(f"{what} lies in a buffer of the layer that this call writes")

    def dense(self, names: Sequence[str], q, layer_idx: int, stream=None) -> None:
        """Projections of the same 8-bit rows into ``self.y``, without their add-ons."""
        self._rows(q, self.shapes[names[0]][0], "q", torch.int8)
        pairs = [self.weights[n][layer_idx] for n in names]
        B.sgmv_dense_q8(self.dtype, [self.y[n] for n in names], q, self.q_scales, [w for w, _ in pairs], [s for _, s in pairs],
                        self.n_tokens, self.shapes[names[0]][0], [self.shapes[n][1] for n in names], self.scratch,
                        self.scratch.numel(), stream)

    def project(self, names: Sequence[str], q, x, layer_idx: int, scale: float = 1.0, stream=None) -> None:
        """Projections of the same rows, ``q`` in 8 bits and ``x`` in 16, and their add-ons, into ``self.y``."""
        if self.add_ons:
            self._rows(x, self.shapes[names[0]][0], "x")
            self._apart(x, [self.y[n] for n in names], "x")  # the add-ons read it after the projections are written
        self.dense(names, q, layer_idx, stream)
        if self.add_ons:
            self.add_lora_group(names, [self.y[n] for n in names], [x] * len(names), layer_idx, scale, stream)

    def norm(self, which: int, x, residual, layer_idx: int, stream=None) -> None:
        """``residual += x`` (in place), its norm into ``self.x`` and ``self.q``; ``which``: 0 attention's, 1 the MLP's.  ``x`` None:
        the residual as it is."""
        for t, what in ((x, "x"), (residual, "residual")):
            if t is not None:
                self._rows(t, self.h, what)
        s = residual if x is None else x
        B.sgmv_rms_norm_q8(self.dtype, self.x, self.q, self.q_scales, None if x is None else residual, s,
                           None if x is None else residual, self.norms[layer_idx][which], self.eps, self.n_tokens, self.h, stream)

    def qkv(self, x, residual, layer_idx: int, scale: float = 1.0, stream=None):
        """Up to attention: norm, q / k / v with their add-ons."""
        self._apart(residual, (self.x, self.y["q"], self.y["k"], self.y["v"]), "residual")
        self.norm(0, x, residual, layer_idx, stream)
        self.project(("q", "k", "v"), self.q, self.x, layer_idx, scale, stream)
        return self.y["q"], self.y["k"], self.y["v"]

    def finish(self, attention, residual, layer_idx: int, scale: float = 1.0, stream=None):
        """From attention's output on: o, norm, gate / up, activation, down.  Returns what the next layer adds to the residual."""
        self._rows(attention, self.h, "attention")
        if residual is not None:
            self._rows(residual, self.h, "residual")  # before anything is enqueued
            self._apart(residual, (self.y["o"], self.x, self.y["gate"], self.y["up"], self.act, self.y["down"]), "residual")
        if self.add_ons:
            self._apart(attention, (self.y["o"],), "attention")
        B.sgmv_quantize_q8(self.dtype, self.q, self.q_scales, attention, self.n_tokens, self.h, stream)
        self.project(("o",), self.q, attention, layer_idx, scale, stream)
        self.norm(1, self.y["o"], residual, layer_idx, stream)
        self.project(("gate", "up"), self.q, self.x, layer_idx, scale, stream)
        B.sgmv_silu_mul_q8(self.dtype, self.act, self.q_ffn, self.q_scales, self.y["gate"], self.y["up"], self.n_tokens, self.ffn,
                           stream)
        self.project(("down",), self.q_ffn, self.act, layer_idx, scale, stream)
        return self.y["down"]

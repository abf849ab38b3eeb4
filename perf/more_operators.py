#!/usr/bin/env python3
"""Attention of a decoder layer over a paged cache held in 4 bits, with what it needs, as cases that can be timed and compared.

Between the q / k / v projections (with their add-ons) and the o projection a served batch runs

  assign   once a step: pages of the cache for every request's new tokens, from the requests' lengths alone; the block
           tables, the slot and the position of every token row, the rows at which the requests start; pages of requests
           that are over go back
  append   rotary positions of q and k, then k and v in 4 bits into the slots; the rows are read back as the values that
           the cache now holds
  attend   causal attention of all rows over their requests' pages: prompts, single tokens, both in one batch

The cache.  pages [n_pages][layers][kv heads][page / 16] tiles; a tile holds 16 positions p of one head, for a head of d values
  8 d bytes   k codes    value j of position p in nibble j % 2 of byte p * d / 2 + j / 2
  8 d bytes   v codes    ... of byte (p / 4) * 2 d + (j / 8) * 16 + (p % 4) * 4 + (j % 8) / 2
  64 bytes    (scale, minimum) of k, 16-bit floats, for every position
  64 bytes    (scale, minimum) of v
A row x in 4 bits: minimum m, scale s = (max - m) / 15 rounded to the 16-bit type, codes c = (x - m) / s rounded to the
nearest, ties to even (0 where s is 0); it stands for c * s + m.

Fields of a case
  op              one of the three
  dtype           "f16" or "bf16"
  heads, kv_heads, d   query heads, heads of the cache, values of a head
  page, layers    positions of a page, layers of the cache (the last one is used)
  prompts, prompt_low, prompt_high    requests that bring a prompt, of so many tokens
  prompt_context  tokens that a prompt's request has in the cache already (up to)
  decodes, rows   requests that bring ``rows`` tokens each (1, or some that a draft model proposed)
  context_low, context_high           tokens that these have in the cache
  over            "assign": requests that are over
  padding         "assign": rows behind the last token
  window          "attend": positions that a row sees at most, 0 for all
  lse             "attend": whether the logarithm of the softmax's sum is wanted
  rope, adjacent  "append": values of a head that are rotated (0: none), pairs (2 i, 2 i + 1) in place of (i, i + rope / 2)
  lengths         seed of the requests' lengths and order
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
_DEFAULTS = dict(op="attend", dtype="f16", heads=32, kv_heads=32, d=128, page=16, layers=2, prompts=0, prompt_low=1, prompt_high=1,
                 prompt_context=0, decodes=0, rows=1, context_low=0, context_high=0, over=0, padding=0, window=0, lse=False, rope=128,
                 adjacent=False, lengths=1)


def _case(**fields):
    return {**_DEFAULTS, **fields}


def listed():
    return [
        # one user's decode step, a short chat so far: the smallest call, launch and host cost
        _case(name="attend_1", decodes=1, context_low=76, context_high=76),
        # the headline decode batch, every request its own adapter, contexts of the paper's layer benchmark
        _case(name="attend_64", decodes=64, context_low=511, context_high=2047),
        # an odd decode batch of a 13B-sized layer whose attention has a window
        _case(name="attend_45_window_bf16", dtype="bf16", heads=40, kv_heads=40, page=64, decodes=45, context_high=4000, window=1024),
        # one request with a very long document, a wide layer with shared heads
        _case(name="attend_long_bf16", dtype="bf16", heads=64, kv_heads=8, page=64, layers=1, decodes=1, context_low=130000,
              context_high=130000),
        # twelve requests that check four drafted tokens each, small heads in odd groups
        _case(name="attend_drafts_d64", heads=14, kv_heads=2, d=64, page=32, decodes=12, rows=4, context_low=90, context_high=3000, lse=True),
        # decode rows next to one prompt, shared heads
        _case(name="attend_mixed_517", kv_heads=8, prompts=1, prompt_low=453, prompt_high=453, decodes=64, context_low=100, context_high=1500),
        # prompts of eight requests
        _case(name="attend_prefill", prompts=8, prompt_low=128, prompt_high=1024),
        # two long prompts, partly in the cache already, of a wide layer: the largest
        _case(name="attend_prefill_wide_bf16", dtype="bf16", heads=64, kv_heads=8, page=64, layers=1, prompts=2, prompt_low=4095,
              prompt_high=4095, prompt_context=1000),
        # one user's decode step
        _case(name="append_1", op="append", decodes=1, context_low=76, context_high=76),
        # prompts of eight requests through a wide layer
        _case(name="append_prefill_bf16", op="append", dtype="bf16", heads=64, kv_heads=8, page=64, layers=1, prompts=8, prompt_low=180,
              prompt_high=1024),
        # the headline decode batch, three requests over
        _case(name="assign_64", op="assign", decodes=64, context_low=511, context_high=2047, over=3),
        # a large batch with prompts in it, in a buffer for more rows
        _case(name="assign_prefill", op="assign", prompts=40, prompt_low=1, prompt_high=1024, prompt_context=500, decodes=960,
              context_high=4000, over=60, padding=777),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _fits(case):
    """Whether a drawn case costs no more than the largest listed ones, also in its plain form, which pads every request."""
    new, old, _ = _lengths(case)
    total, costs = new + old, work(case)
    if case["op"] == "assign":
        return len(new) <= 1100 and int(new.sum()) + case["padding"] <= 23000
    cached = int(total.sum()) * case["kv_heads"] * case["layers"]
    if case["op"] == "append":
        return costs["bytes"] <= 1.8e8 and cached <= 6e6
    padded = len(new) * int(total.max())
    return (costs["flops"] <= 5.8e11 and costs["bytes"] <= 3.8e8 and cached <= 8e6 and padded * case["kv_heads"] * case["d"] <= 7e8
            and padded * case["heads"] * int(new.max()) <= 2e9)


def draw(rng):
    while True:
        c = _case(op=rng.choice(("attend", "attend", "attend", "attend", "append", "append", "assign")), dtype=rng.choice(("f16", "bf16")),
                  kv_heads=rng.choice((1, 2, 4, 5, 8, 8, 16, 32, 40)), d=rng.choice((64, 128, 128)), page=rng.choice((16, 16, 32, 64, 128)),
                  layers=rng.randint(1, 3), lengths=rng.randrange(1 << 20))
        c["heads"] = c["kv_heads"] * rng.choice((1, 1, 2, 4, 5, 7, 8)) if c["kv_heads"] < 16 else c["kv_heads"]
        kind = rng.choice(("decode", "decode", "prompt", "mixed"))
        if kind != "prompt":
            c["decodes"] = _log_uniform(rng, 1, 1200 if c["op"] == "assign" else 128)
            c["rows"] = rng.choice((1, 1, 1, 1, 2, 3, 5))
            c["context_high"] = _log_uniform(rng, 1, 131072 if c["decodes"] < 3 else 6000)
            c["context_low"] = rng.choice((0, c["context_high"] // 3, c["context_high"]))
        if kind != "decode":
            c["prompts"] = 1 if kind == "mixed" else _log_uniform(rng, 1, 16)
            c["prompt_high"] = _log_uniform(rng, 1, 5000)
            c["prompt_low"] = rng.choice((1, c["prompt_high"] // 8 + 1, c["prompt_high"]))
            c["prompt_context"] = rng.choice((0, 0, _log_uniform(rng, 1, 4000)))
        if c["op"] == "assign":
            c["over"] = rng.choice((0, 0, 1, 7, 50))
            c["padding"] = rng.choice((0, 5, 300))
        elif c["op"] == "append":
            c["rope"] = rng.choice((0, c["d"], c["d"], c["d"] // 2))
            c["adjacent"] = c["rope"] > 0 and rng.random() < 0.4
        else:
            c["window"] = rng.choice((0, 0, 0, _log_uniform(rng, 1, 4096)))
            c["lse"] = rng.random() < 0.3
        if _fits(c):
            return c


def _lengths(case):
    """Tokens that the requests bring and have, in the order of the batch, and which of them are over."""
    rs = np.random.RandomState(case["lengths"])
    prompts, decodes, over = case["prompts"], case["decodes"], case["over"]
    new = np.concatenate([rs.randint(case["prompt_low"], case["prompt_high"] + 1, prompts), np.full(decodes, case["rows"]), np.zeros(over, int)])
    old = np.concatenate([rs.randint(0, case["prompt_context"] + 1, prompts),
                          rs.randint(case["context_low"], case["context_high"] + 1, decodes),
                          rs.randint(0, max(case["context_high"], case["prompt_high"]) + 1, over)])
    ended = np.arange(len(new)) >= prompts + decodes
    order = rs.permutation(len(new))
    return new[order].astype(np.int64), old[order].astype(np.int64), ended[order]


def _visible(case):
    """(pairs of a row and a position it sees, positions of the cache that some row sees) of the batch."""
    new, old, _ = _lengths(case)
    pairs = seen = 0
    for n, before in zip(new.tolist(), old.tolist()):
        ends = before + 1 + np.arange(n)
        sees = np.minimum(ends, case["window"]) if case["window"] else ends
        pairs += int(sees.sum())
        seen += int(ends[-1] - (ends[0] - sees[0])) if n else 0
    return pairs, seen


def work(case):
    new, old, ended = _lengths(case)
    rows, d, h, n = int(new.sum()), case["d"], case["heads"], case["kv_heads"]
    held = n * 2 * (d // 2 + 4)  # bytes of a position
    if case["op"] == "attend":
        pairs, seen = _visible(case)
        pages = int((-(-(new + old) // case["page"])).sum())
        return {"bytes": seen * held + 4 * rows * h * d + 4 * pages + 8 * len(new) + (4 * rows * h if case["lse"] else 0), "flops": 4 * pairs * h * d}
    if case["op"] == "append":
        turned = rows * h * d * 4 if case["rope"] else 0
        return {"bytes": rows * (4 * n * d + 2 * held + 4 * n * d + 8 + 4 * case["rope"]) + turned,
                "flops": rows * d * (3 * (h + n) * (case["rope"] > 0) + 10 * n)}
    page = case["page"]
    moved = int((-(-old[ended] // page)).sum() + (-(-(new + old)[~ended] // page) - -(-old[~ended] // page)).sum())
    return {"bytes": 4 * (4 * len(new) + 2 * rows + 2 * case["padding"] + 2 * moved), "flops": 4 * rows}


def _tile_bytes(case):
    return 16 * case["d"] + 128


def _quantize(x, t):
    """(codes, scales, minima) of rows of 16-bit values, the last two rounded to ``t`` and as fp32."""
    m, top = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((top - m) / torch.full_like(m, 15.0)).to(t).float()
    c = torch.where(s > 0, torch.round((x - m) / s), torch.zeros_like(x)).clamp_(0, 15)
    return c, s, m


def _nibbles(c):
    c = c.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _pack(k, v, t):
    """Tiles of the cache from rows [tiles, 16, d] of k and v."""
    parts = []
    for x, is_v in ((k, False), (v, True)):
        c, s, m = _quantize(x.to(t).float(), t)
        b, n = _nibbles(c), c.shape[0]
        if is_v:
            b = b.view(n, 4, 4, -1, 4).permute(0, 1, 3, 2, 4)
        parts.append((b.reshape(n, -1), torch.cat((s, m), -1).to(t).contiguous().view(torch.uint8).reshape(n, -1)))
    return torch.cat((parts[0][0], parts[1][0], parts[0][1], parts[1][1]), 1)


def _unpack(tiles, d, t):
    """(k, v) as fp32 [tiles, 16, d]: the values that the tiles stand for."""
    n, codes = tiles.shape[0], 8 * d
    k = tiles[:, :codes].reshape(n, 16, d // 2)
    v = tiles[:, codes:2 * codes].reshape(n, 4, d // 8, 4, 4).permute(0, 1, 3, 2, 4).reshape(n, 16, d // 2)
    params = tiles[:, 2 * codes:].contiguous().view(t).float().view(n, 2, 16, 2)
    return [torch.stack((b & 15, b >> 4), -1).view(n, 16, d).float() * params[:, i, :, :1] + params[:, i, :, 1:] for i, b in ((0, k), (1, v))]


def _rows(gen, *shape):
    """Keys or values of a language model: normal, with a few channels that are larger in every row."""
    wide = 1.0 + 4.0 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.03)
    return torch.randn(*shape, generator=gen, device="cuda") * wide


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    new, old, ended = _lengths(case)
    rows, page, t = int(new.sum()), case["page"], TORCH[case["dtype"]]
    h, n, d = case["heads"], case["kv_heads"], case["d"]

    def ints(values):
        return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")

    s = {"case": case, "t": t, "n_reqs": len(new)}
    assigning = case["op"] == "assign"
    # pages that the requests hold, in any order; their tables are wider than today's longest request
    had = -(-old // page) if assigning else -(-(new + old) // page)
    width = int((-(-(new + old) // page)).max()) + 2
    spare = int((-(-(new + old) // page)).sum()) + 3 if assigning else 0
    n_pages = int(had.sum()) + spare
    shuffled = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    place = torch.arange(width, device="cuda")[None] < ints(had)[:, None]
    at = torch.cumsum(place.view(-1), 0).view_as(place) - 1
    s["tables"] = torch.where(place, shuffled[at.clamp_min(0)], torch.full_like(shuffled[at.clamp_min(0)], -1))
    s["n_pages"], s["width"] = n_pages, width
    n_rows = rows + case["padding"]
    s["n_rows"] = n_rows
    s["max_q"], s["max_kv"] = int(new.max()), int((new + old).max())
    s["q_starts"] = ints(np.concatenate(([0], np.cumsum(new))))
    s["slots"], s["positions"] = ints(np.full(n_rows, -1)), ints(np.full(n_rows, -1))
    if assigning:
        s["new_lens"], s["old_lens"] = ints(np.where(ended, -1, new)), ints(old)
        s["lens"] = torch.zeros_like(s["old_lens"])
        s["free_pages"] = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        s["free_pages"][:spare] = shuffled[n_pages - spare:]
        s["free_count"], s["free_count_out"] = ints([spare]), ints([0])
        s["status"] = ints([0, 0])
        return s
    s["lens"] = ints(new + old)
    req = np.repeat(np.arange(len(new)), new)
    pos = np.arange(rows) - np.repeat(np.cumsum(new) - new, new) + old[req]
    s["positions"] = ints(pos)
    where = torch.tensor(req, device="cuda"), torch.tensor(pos // page, device="cuda")
    s["slots"] = s["tables"][where] * page + s["positions"] % page
    tiles = page // 16
    s["pages"] = torch.zeros(n_pages, case["layers"], n, tiles, _tile_bytes(case), dtype=torch.uint8, device="cuda")
    s["q"] = _rows(gen, rows, h, d).to(t)
    if case["op"] == "append":
        s["k"], s["v"] = _rows(gen, rows, n, d).to(t), _rows(gen, rows, n, d).to(t)
        s["q_out"], s["k_out"], s["v_out"] = (torch.empty_like(s[name]) for name in "qkv")
        if case["rope"]:
            half = case["rope"] // 2
            angles = np.arange(s["max_kv"])[:, None] * 10000.0 ** (-np.arange(half) / half)
            s["rope"] = torch.tensor(np.concatenate((np.cos(angles), np.sin(angles)), 1), dtype=torch.float32, device="cuda")
        return s
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(rows, h, dtype=torch.float32, device="cuda") if case["lse"] else None
    layer = s["pages"][:, -1]
    step = max(1, (1 << 27) // (n * tiles * 16 * d))
    for first in range(0, n_pages, step):
        shape = (min(step, n_pages - first) * n * tiles, 16, d)
        layer[first:first + step] = _pack(_rows(gen, *shape), _rows(gen, *shape), t).view(-1, n, tiles, _tile_bytes(case))
    s["scale"] = 1.0 / math.sqrt(d)
    s["scratch"] = torch.empty(128 << 20, dtype=torch.uint8, device="cuda")  # what a program keeps for its longest step
    return s


def _plain_assign(s):
    page, width, n_pages = s["case"]["page"], s["width"], s["n_pages"]
    new, old, tables = s["new_lens"].long(), s["old_lens"].long(), s["tables"].long()
    over = new < 0
    rows = new.clamp_min(0)
    lens = torch.where(over, torch.zeros_like(old), old + rows)
    held, column = (old + page - 1) // page, torch.arange(width, device="cuda")
    # released pages onto the stack, then the needed ones off its top
    back = over[:, None] & (column < held[:, None])
    order = torch.cumsum(back.view(-1), 0)
    to = torch.where(back.view(-1), s["free_count"] + order - 1, torch.full_like(order, n_pages))
    free = torch.cat((s["free_pages"].long(), held[:1])).scatter(0, to, tables.view(-1))[:-1]
    top = s["free_count"].long() + order[-1]
    more = ~over[:, None] & (column >= held[:, None]) & (column * page < lens[:, None])
    count = torch.cumsum(more.view(-1), 0)
    taken = free[(top - count).clamp(0, n_pages - 1)].view_as(tables)
    tables = torch.where(more, taken, tables)
    ends = torch.cumsum(rows, 0)
    starts = torch.cat((torch.zeros_like(ends[:1]), ends))
    t = torch.arange(s["n_rows"], device="cuda")
    live = t < ends[-1]
    req = torch.searchsorted(ends, t, right=True).clamp_max(len(new) - 1)
    pos = lens[req] - ends[req] + t
    slot = tables[req, (pos // page).clamp(0, width - 1)] * page + pos % page
    none = torch.full_like(t, -1)
    result = {"lens": lens, "tables": tables, "free_pages": free, "free_count": top - count[-1:], "q_starts": starts,
              "slots": torch.where(live, slot, none), "positions": torch.where(live, pos, none), "status": torch.zeros_like(top[:1]).repeat(2)}
    return {name: x.to(torch.int32) for name, x in result.items()}


def _turned(s, x):
    """Rows with their first ``rope`` values rotated by their positions, rounded to 16 bits: every product and sum in fp32."""
    dim, t = s["case"]["rope"], s["t"]
    if not dim:
        return x
    cos, sin = s["rope"][s["positions"].long()][:, None].chunk(2, -1)
    x = x.float()
    a, b = (x[..., 0:dim:2], x[..., 1:dim:2]) if s["case"]["adjacent"] else (x[..., :dim // 2], x[..., dim // 2:dim])
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.stack((a, b), -1).flatten(-2) if s["case"]["adjacent"] else torch.cat((a, b), -1)
    return torch.cat((both, x[..., dim:]), -1).to(t)


def _plain_append(s):
    result = {"q": _turned(s, s["q"]) if s["case"]["rope"] else None}
    for name, x in (("k", _turned(s, s["k"])), ("v", s["v"])):
        c, scale, m = _quantize(x.float(), s["t"])
        result[name] = (c * scale + m).to(s["t"])
    return result


def _plain_attend(s):
    case, t, page, n, d = s["case"], s["t"], s["case"]["page"], s["case"]["kv_heads"], s["case"]["d"]
    group, reqs = case["heads"] // n, s["n_reqs"]
    pages = -(-s["max_kv"] // page)
    longest = pages * page
    # every request's pages side by side, [requests, kv heads, positions, d]
    tables = s["tables"][:, :pages].long().clamp_min(0)
    tiles = s["pages"][tables, -1].permute(0, 2, 1, 3, 4).reshape(-1, _tile_bytes(case))
    k, v = (x.view(reqs, n, longest, d) for x in _unpack(tiles, d, t))
    starts, lens = s["q_starts"].long(), s["lens"].long()
    row = torch.arange(s["max_q"], device="cuda")
    live = row < (starts[1:] - starts[:-1])[:, None]
    at = (starts[:-1, None] + row).clamp_max(s["n_rows"] - 1)
    q = s["q"].float()[at].view(reqs, s["max_q"], n, group, d).permute(0, 2, 3, 1, 4).reshape(reqs, n, group * s["max_q"], d)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).view(reqs, n, group, s["max_q"], longest)
    p = torch.arange(longest, device="cuda")
    last = (lens - (starts[1:] - starts[:-1]))[:, None] + row  # the position of a row's own token
    sees = (p <= last[..., None]) & (p < lens[:, None, None])
    if case["window"]:
        sees &= p > last[..., None] - case["window"]
    x.masked_fill_(~sees[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(reqs, n, group * s["max_q"], longest), v).view(reqs, n, group, s["max_q"], d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out)).permute(0, 3, 1, 2, 4).reshape(reqs, s["max_q"], n * group, d)
    to = torch.where(live, at, torch.full_like(at, s["n_rows"])).view(-1)
    result = {"out": torch.empty(s["n_rows"] + 1, n * group, d, dtype=t, device="cuda").index_copy_(0, to, out.flatten(0, 1).to(t))[:-1], "lse": None}
    if case["lse"]:
        lse = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(-1, n * group)
        result["lse"] = torch.empty(s["n_rows"] + 1, n * group, device="cuda").index_copy_(0, to, lse)[:-1]
    return result


def _handles(s):
    """What a program keeps for its batch: the descriptors of the cache, the batch and the rotation."""
    from paper_2310_18547_amd import binding as B
    case = s["case"]
    cache = B.make_kv_cache(B.F16 if case["dtype"] == "f16" else B.BF16, case["d"], case["kv_heads"], case["layers"], case["page"],
                            s["n_pages"], pages=s.get("pages"))
    batch = B.make_kv_batch(s["n_reqs"], s["n_rows"], s["width"], s["q_starts"], s["lens"], s["tables"], s["slots"], s["positions"],
                            max_q_len=s["max_q"], max_kv_len=s["max_kv"])
    rope = B.make_rope(s["rope"], s["max_kv"], case["rope"], int(case["adjacent"])) if "rope" in s else None
    return B, cache, batch, rope


def _calls(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    B, cache, batch, rope = s["handles"]
    case = s["case"]
    layer, h, n, d = case["layers"] - 1, case["heads"], case["kv_heads"], case["d"]
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "assign":
        B.sgmv_kv_assign(cache, batch, s["new_lens"], s["old_lens"], s["free_pages"], s["free_count"], s["free_count_out"], s["status"], stream)
        return {"lens": s["lens"], "tables": s["tables"], "free_pages": s["free_pages"], "free_count": s["free_count_out"],
                "q_starts": s["q_starts"], "slots": s["slots"], "positions": s["positions"], "status": s["status"]}
    if case["op"] == "append":
        q_out, q = (s["q_out"], s["q"]) if rope is not None else (None, None)
        B.sgmv_kv_append_q4(cache, batch, layer, q_out, q, s["k"], s["v"], h, h * d, h * d, n * d, rope, stream)
        B.sgmv_kv_read_q4(cache, layer, s["k_out"], s["v_out"], n * d, s["slots"], s["n_rows"], stream)
        return {"q": q_out, "k": s["k_out"], "v": s["v_out"]}
    B.sgmv_attention_q4(cache, batch, layer, s["out"], s["lse"], s["q"], h, h * d, h * d, s["scale"], 1, case["window"], s["scratch"],
                        s["scratch"].numel(), stream)
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _calls(state)
    op = state["case"]["op"]
    return _plain_assign(state) if op == "assign" else _plain_append(state) if op == "append" else _plain_attend(state)


def exact(case, seed):
    if case["op"] == "assign":
        return None  # whole numbers only
    s = prepare(case, seed)
    t, d = s["t"], case["d"]
    new, old, _ = _lengths(case)
    if case["op"] == "append":
        result = {}
        for name in "qkv":
            x = s[name].to(torch.float64)
            if name != "v" and case["rope"]:
                half = case["rope"] // 2
                table = s["rope"][s["positions"].long()].to(torch.float64)
                turn = torch.complex(table[:, :half], table[:, half:]).view(-1, 1, half)
                first = slice(0, case["rope"], 2) if case["adjacent"] else slice(0, half)
                second = slice(1, case["rope"], 2) if case["adjacent"] else slice(half, case["rope"])
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
                if name == "k":
                    x = x.to(t).to(torch.float64)  # the cache quantises 16-bit rows
            if name == "q":
                result[name] = x if case["rope"] else None
                continue
            low = x.min(-1, keepdim=True).values
            step = ((x.max(-1, keepdim=True).values - low) / 15).to(t).to(torch.float64)
            levels = torch.round(torch.nan_to_num((x - low) / step, nan=0.0, posinf=0.0)).clamp(0, 15)
            result[name] = low + step * levels
        return result
    result = {"out": torch.zeros(s["n_rows"], case["heads"], d, dtype=torch.float64, device="cuda"),
              "lse": torch.zeros(s["n_rows"], case["heads"], dtype=torch.float64, device="cuda") if case["lse"] else None}
    shifts = torch.tensor([0, 4], dtype=torch.uint8, device="cuda")
    first, codes, group = 0, 8 * d, case["heads"] // case["kv_heads"]
    for r, (n, before) in enumerate(zip(new.tolist(), old.tolist())):
        if n == 0:
            continue
        total = n + before
        held = s["pages"][s["tables"][r, :-(-total // case["page"])].long(), -1].transpose(0, 1)  # [heads, pages, tiles, bytes]
        where = torch.arange(total, device="cuda")
        span = where[None] - (before + torch.arange(n, device="cuda"))[:, None]  # 0 at a row's own token
        hidden = (span > 0) | ((span <= -case["window"]) if case["window"] else (span > 0))
        for g in range(case["kv_heads"]):
            tiles = held[g].reshape(-1, _tile_bytes(case))
            pairs = tiles[:, 2 * codes:].contiguous().view(t).to(torch.float64).view(-1, 2, 16, 2)
            k = tiles[:, :codes].reshape(-1, 16, d // 2)
            v = tiles[:, codes:2 * codes].reshape(-1, 4, d // 8, 4, 4).transpose(2, 3).reshape(-1, 16, d // 2)
            k, v = (((b[..., None] >> shifts) & 15).view(-1, 16, d).to(torch.float64) * pairs[:, i, :, 0, None] + pairs[:, i, :, 1, None]
                    for i, b in enumerate((k, v)))
            k, v = k.reshape(-1, d)[:total], v.reshape(-1, d)[:total]
            q = s["q"][first:first + n, g * group:(g + 1) * group].to(torch.float64)
            x = torch.matmul(q.reshape(-1, d), k.t().contiguous()).view(n, group, total) * s["scale"]
            x = x.masked_fill(hidden[:, None], -math.inf)
            result["out"][first:first + n, g * group:(g + 1) * group] = torch.matmul(torch.softmax(x, -1).view(-1, total), v).view(n, group, d)
            if case["lse"]:
                result["lse"][first:first + n, g * group:(g + 1) * group] = torch.logsumexp(x, -1)
        first += n
    return result

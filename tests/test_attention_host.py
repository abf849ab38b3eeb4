"""The paged 4-bit cache's calls without a GPU: what they refuse, sizes, and which kernels a call resolves to."""
import ctypes

import pytest
import torch  # noqa: F401  (before the library: a process has one HIP runtime, torch's)

import paper_2310_18547_amd as sg

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, RANGE = 0, 1, 2, 3, 4, 6
NAMES = ("pages", "q_out", "q", "k", "v", "out", "lse", "q_starts", "kv_lens", "tables", "slots", "positions", "rope", "workspace", "new", "old",
         "free", "count", "count_out", "status")
AT = {name: (i + 1) << 24 for i, name in enumerate(NAMES)}  # addresses that are never dereferenced on these paths


def cache(**k):
    a = dict(dtype=sg.F16, head_dim=128, n_kv_heads=2, num_layers=2, page_size=16, n_pages=8, pages=AT["pages"], page_stride=0)
    a.update(k)
    return sg.make_kv_cache(**a)


def batch(**k):
    a = dict(n_reqs=3, n_tokens=4, table_width=5, **{n: AT[n] for n in ("q_starts", "kv_lens", "tables", "slots", "positions")})
    a.update(k)
    return sg.make_kv_batch(**a)


def assign(c=None, b=None, **k):
    a = {**AT, **k}
    return sg.sgmv_kv_assign(c or cache(), b or batch(), a["new"], a["old"], a["free"], a["count"], a["count_out"], a["status"], check=False)


def append(c=None, b=None, layer=0, heads=4, q_out_stride=512, q_stride=512, kv_stride=256, rope=(50, 128, 0), **k):
    a = {**AT, **k}
    return sg.sgmv_kv_append_q4(c or cache(), b or batch(), layer, a["q_out"], a["q"], a["k"], a["v"], heads, q_out_stride, q_stride, kv_stride,
                                None if rope is None else sg.make_rope(a["rope"], *rope), check=False)


def read(c=None, layer=0, stride=256, n=4, **k):
    a = {**AT, **k}
    return sg.sgmv_kv_read_q4(c or cache(), layer, a["k"], a["v"], stride, a["slots"], n, check=False)


def attention(c=None, b=None, layer=0, heads=4, out_stride=512, q_stride=512, scale=0.1, causal=1, window=0, nbytes=1 << 20, **k):
    a = {**AT, **k}
    return sg.sgmv_attention_q4(c or cache(), b or batch(), layer, a["out"], a["lse"], a["q"], heads, out_stride, q_stride, scale, causal, window,
                                a["workspace"], nbytes, check=False)


CALLS = [assign, append, read, attention]


@pytest.mark.parametrize("call", CALLS)
def test_caches_that_are_refused(call):
    for field, values in (("dtype", (2, -1)), ("head_dim", (8, 96, 256)), ("page_size", (8, 24, 512, 48))):
        for v in values:
            assert call(cache(**{field: v})) == UNSUPPORTED, (field, v)
            assert sg.sgmv_kv_page_bytes(cache(**{field: v})) == 0
    for field in ("head_dim", "n_kv_heads", "num_layers", "page_size", "n_pages"):
        for v in (0, -1):
            assert call(cache(**{field: v})) == SHAPE, (field, v)
    assert call(cache(n_kv_heads=65537)) == UNSUPPORTED
    assert call(cache(n_pages=1 << 27)) == UNSUPPORTED  # positions past 32 bits
    if call is assign:
        return
    for layer in (-1, 2):
        assert call(layer=layer) == RANGE
    assert call(cache(pages=None)) == NULL
    assert call(cache(pages=AT["pages"] + 8)) == ALIGN
    size = sg.sgmv_kv_page_bytes(cache())
    assert size == 2 * 2 * (16 * 128 + 128)
    assert call(cache(page_stride=size - 16)) == SHAPE and call(cache(page_stride=size + 8)) == ALIGN
    assert call(cache(page_stride=1 << 62)) == SHAPE


@pytest.mark.parametrize("call", [assign, append, attention])
def test_batches_that_are_refused(call):
    for field in ("n_reqs", "n_tokens", "table_width", "max_q_len", "max_kv_len"):
        assert call(b=batch(**{field: -1})) == SHAPE, field
    assert call(b=batch(table_width=1 << 27)) == UNSUPPORTED
    assert call(b=batch(n_reqs=0, q_starts=None, kv_lens=None, tables=None, slots=None, positions=None)) == OK
    if call is not assign:
        assert call(b=batch(n_tokens=0, q_starts=None, kv_lens=None, tables=None, slots=None, positions=None)) == OK


def test_pointers_that_are_missing_or_not_aligned():
    for name in ("new", "old", "free", "count", "count_out", "status"):
        assert assign(**{name: None}) == NULL and assign(**{name: AT[name] + 2}) == ALIGN, name
    for name in ("q_starts", "kv_lens", "tables", "slots", "positions"):
        assert assign(b=batch(**{name: None})) == NULL and assign(b=batch(**{name: AT[name] + 2})) == ALIGN, name
    for name in ("k", "v"):
        assert append(**{name: None}) == NULL and append(**{name: AT[name] + 8}) == ALIGN
        assert read(**{name: AT[name] + 8}) == ALIGN
    assert append(q=None) == NULL and append(q_out=None) == NULL and append(q=AT["q"] + 2) == ALIGN and append(q_out=AT["q_out"] + 8) == ALIGN
    assert append(b=batch(slots=None)) == NULL and append(b=batch(positions=None)) == NULL
    assert read(k=None, v=None) == NULL and read(slots=None) == NULL and read(slots=AT["slots"] + 1) == ALIGN
    for name in ("out", "q"):
        assert attention(**{name: None}) == NULL and attention(**{name: AT[name] + 8}) == ALIGN
    for name in ("q_starts", "kv_lens", "tables"):
        assert attention(b=batch(**{name: None})) == NULL and attention(b=batch(**{name: AT[name] + 2})) == ALIGN
    assert attention(lse=AT["lse"] + 2) == ALIGN and attention(workspace=AT["workspace"] + 128) == ALIGN


def test_sizes_that_are_refused():
    assert append(heads=0) == SHAPE and append(heads=65537, q_stride=1 << 24, q_out_stride=1 << 24) == UNSUPPORTED
    for name in ("q_out_stride", "q_stride", "kv_stride"):
        assert append(**{name: 248}) == SHAPE and append(**{name: 516}) == SHAPE and append(**{name: -512}) == SHAPE and append(**{name: 1 << 61}) == SHAPE
    assert append(rope=None) == SHAPE  # q without a rotation
    assert append(rope=None, q=None, q_out=None, k=None) == NULL
    assert append(rope=(-1, 128, 0)) == SHAPE and append(rope=(5, 0, 0)) == SHAPE and append(rope=(5, 8, 0)) == UNSUPPORTED
    assert append(rope=(5, 144, 0)) == UNSUPPORTED and append(cache(head_dim=64), kv_stride=256, rope=(5, 128, 0)) == UNSUPPORTED
    assert read(n=-1) == SHAPE and read(n=0, k=None, v=None, slots=None) == OK and read(stride=128) == SHAPE
    assert attention(heads=3) == SHAPE and attention(heads=0) == SHAPE and attention(heads=-2) == SHAPE and attention(window=-1) == SHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attention(scale=scale) == UNSUPPORTED
    for name in ("out_stride", "q_stride"):
        assert attention(**{name: 504}) == SHAPE and attention(**{name: 516}) == SHAPE
    assert attention(b=batch(n_tokens=1 << 30)) == UNSUPPORTED  # rows x heads past 32 bits
    assert attention(nbytes=(1 << 64) - 1) == SHAPE


def test_buffers_that_overlap_are_refused():
    written = ("q_starts", "kv_lens", "tables", "slots", "positions")
    for name in written:
        for other in (*written, "new", "old", "free", "count", "count_out", "status"):
            if other != name and (name, other) != ("kv_lens", "old"):
                assert assign(b=batch(**{name: AT[other]})) == SHAPE, (name, other)
    assert assign(count_out=AT["status"]) == SHAPE and assign(old=AT["kv_lens"] + 4) == SHAPE
    # q's rows over k's, unless they lie side by side in one row
    assert append(q_out=AT["k"]) == SHAPE and append(q_out=AT["q"] + 16) == SHAPE and append(q_out=AT["q"], q_out_stride=520) == SHAPE
    for name in ("slots", "positions"):
        assert append(q_out=AT[name] - 64) == SHAPE
    assert append(q_out=AT["rope"]) == SHAPE
    for name in ("q", "q_out", "k", "v"):
        assert append(**{name: AT["pages"] + 8 * sg.sgmv_kv_page_bytes(cache()) - 16}) == SHAPE, name
    fused = dict(q_out=AT["q"], q=AT["q"], q_out_stride=1024, q_stride=1024, kv_stride=1024, v=AT["q"] + 2 * 768)
    assert append(**fused, k=AT["q"] + 2 * 504) == SHAPE
    assert append(**fused, k=AT["q"] + 2 * 1016) == SHAPE  # its end in the next row's q
    assert read(k=AT["v"] + 16) == SHAPE and read(k=AT["pages"]) == SHAPE and read(v=AT["slots"] - 16) == SHAPE
    long = batch(table_width=400)  # in slices
    for name in ("q", "lse", "workspace", "pages", "q_starts", "kv_lens", "tables"):
        assert attention(b=long, out=AT[name]) == SHAPE, name
    for name in ("q", "pages", "q_starts", "kv_lens", "tables"):
        assert attention(lse=AT[name]) == SHAPE, name
        assert attention(b=long, workspace=AT[name]) == SHAPE, name


def test_descriptors_of_another_kind_raise():
    for wrong in (None, 5, batch()):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            sg.sgmv_kv_assign(wrong, batch(), 1, 1, 1, 1, 1, 1)
    with pytest.raises((TypeError, ctypes.ArgumentError)):
        sg.sgmv_attention_q4(cache(), cache(), 0, 1, 1, 1, 4, 512, 512, 0.1)
    with pytest.raises((TypeError, ctypes.ArgumentError)):
        sg.sgmv_kv_append_q4(cache(), batch(), 0, 1, 1, 1, 1, 4, 512, 512, 256, batch())
    with pytest.raises((TypeError, ctypes.ArgumentError)):
        sg.sgmv_kv_read_q4(cache(), 0, 1, 1, "256", 1, 4)
    with pytest.raises(sg.SgmvError):
        sg.sgmv_kv_read_q4(cache(), 9, 1, 1, 256, 1, 4)


def test_plans_and_workspaces():
    c = cache(n_kv_heads=32, n_pages=100000)
    many = batch(n_reqs=64, n_tokens=64, table_width=128, max_q_len=1, max_kv_len=2048)
    one = batch(n_reqs=1, n_tokens=1, table_width=8192, max_q_len=1, max_kv_len=131072)
    for b in (many, one):
        need = sg.sgmv_attention_workspace_bytes(c, b, 32)
        plan = sg.sgmv_plan_attention_q4(c, b, 32, 0, AT["workspace"], need)
        assert (plan.slices > 1) == (need > 0) and plan.launches == (2 if need else 1)
        assert need == b.n_tokens * 32 * (4 * 128 + 8) * plan.slices * (plan.slices > 1)
        without = sg.sgmv_plan_attention_q4(c, b, 32)
        assert without.slices == 1 and without.launches == 1
        half = sg.sgmv_plan_attention_q4(c, b, 32, 0, AT["workspace"], need // 2)
        assert half.slices <= max(1, plan.slices // 2)
    assert sg.sgmv_plan_attention_q4(c, one, 32, 0, AT["workspace"], 1 << 30).slices > 8
    assert sg.sgmv_attention_workspace_bytes(c, batch(n_reqs=1, n_tokens=1, table_width=1), 32) == 0
    assert sg.sgmv_attention_workspace_bytes(c, batch(n_reqs=0), 32) == 0 and sg.sgmv_attention_workspace_bytes(c, batch(), 33) == 0
    rc, _ = sg.sgmv_plan_attention_q4(c, batch(), 33, check=False)
    assert rc == SHAPE
    assert sg.sgmv_plan_attention_q4(c, batch(n_tokens=0), 32).launches == 0


def test_structs_match_the_header():
    assert ctypes.sizeof(sg.SgmvKvCache) == 40 and ctypes.sizeof(sg.SgmvKvBatch) == 64 and ctypes.sizeof(sg.SgmvRope) == 24

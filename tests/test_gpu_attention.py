"""The paged 4-bit cache and attention over it on the GPU, against plain Python and 64 bits."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2310_18547_amd as sg
from backbone_reference import round16
from helpers import decode64

pytestmark = pytest.mark.gpu

CODE = {"f16": sg.F16, "bf16": sg.BF16}
KIND = {"f16": torch.float16, "bf16": torch.bfloat16}


def dev(a, dtype=None):
    return torch.tensor(np.ascontiguousarray(a), device="cuda", dtype=dtype)


def ints(a):
    return dev(np.asarray(a, np.int64), torch.int32)


def bits16(a, dtype):
    """16-bit patterns on the device as a tensor of their type."""
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(KIND[dtype])


def host16(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def host(t):
    return t.cpu().numpy()


def normal(rng, shape, dtype, scale=1.0):
    x = rng.standard_normal(shape) * scale * np.where(rng.random(shape[-1]) < 0.05, 4.0, 1.0)
    return round16(x.astype(np.float32), dtype)


class Cache:
    """A cache on the device and the descriptor; pages hold a pattern that no call writes."""

    def __init__(self, dtype, d, heads, layers, page, n_pages, fill=0xA5, pad=0):
        self.dtype, self.d, self.heads, self.layers, self.page, self.n_pages = dtype, d, heads, layers, page, n_pages
        size = sg.sgmv_kv_page_bytes(sg.make_kv_cache(CODE[dtype], d, heads, layers, page, n_pages))
        assert size == layers * heads * page // 16 * (16 * d + 128)
        self.store = torch.full((n_pages, size + pad), fill, dtype=torch.uint8, device="cuda")
        self.size = size
        self.c = sg.make_kv_cache(CODE[dtype], d, heads, layers, page, n_pages, self.store, size + pad if pad else 0)

    def bytes(self):
        return host(self.store[:, :self.size]).reshape(self.n_pages, self.layers, self.heads, self.page // 16, 16 * self.d + 128)

    def put(self, pages):
        self.store[:, :self.size] = dev(pages.bytes.reshape(self.n_pages, -1))

    def reference(self, fill=0xA5):
        return ref.Pages(self.n_pages, self.layers, self.heads, self.page, self.d, self.dtype, fill)


def rope_table(rows, dim):
    angle = np.arange(rows)[:, None] * 100.0 ** (-np.arange(dim // 2) / (dim // 2))
    return np.concatenate((np.cos(angle), np.sin(angle)), 1).astype(np.float32)


# ---------------------------------------------------------------------------------------------- append and read

def append_case(dtype, d, heads, kv_heads, page, n, dim, adjacent, seed=0, pad=0, fused=False, special=True, slots=None):
    rng = np.random.default_rng(seed)
    n_pages, layers = n // page + 3, 2
    cache = Cache(dtype, d, kv_heads, layers, page, n_pages, pad=pad)
    q, k, v = (normal(rng, (n, h, d), dtype) for h in (heads, kv_heads, kv_heads))
    if special:  # rows of one value, of the largest ones, of the smallest, of what is not finite
        top = round16(np.float32([3e38 if dtype == "bf16" else 65504.0]), dtype)[0]
        for i, row in enumerate((k, v)):
            row[0 % n, 0] = round16(np.float32([0.3]), dtype)[0]
            row[1 % n, 0, ::2], row[1 % n, 0, 1::2] = top, top | 0x8000
            row[2 % n, 0] = rng.integers(0, 5, d)
            row[3 % n, 0, 3 + i] = 0x7F80 if dtype == "bf16" else 0x7C00
            row[4 % n, 0, d - 1] = 0x7FFF
            row[5 % n, 0] = 0
    if slots is None:
        slots = rng.permutation(n_pages * page)[:n]
    positions = rng.integers(0, 50, n)
    table = rope_table(50, dim) if dim else None
    batch_slots, batch_positions = ints(slots), ints(positions)
    b = sg.make_kv_batch(3, n, 1, None, None, None, batch_slots, batch_positions)
    if fused:
        both = torch.zeros(n, (heads + 2 * kv_heads) * d + 8, dtype=KIND[dtype], device="cuda")
        parts = [both[:, :heads * d], both[:, heads * d:(heads + kv_heads) * d], both[:, (heads + kv_heads) * d:-8]]
        for part, x in zip(parts, (q, k, v)):
            part.copy_(bits16(x.reshape(n, -1), dtype))
        dq, dk, dv = parts
        stride = kv_stride = both.shape[1]
        out = dq
    else:
        dq, dk, dv = (bits16(x, dtype) for x in (q, k, v))
        stride, kv_stride = heads * d, kv_heads * d
        out = torch.zeros_like(dq)
    keep = dev(table) if dim else None
    rope = sg.make_rope(keep, 50, dim, adjacent) if dim else None
    sg.sgmv_kv_append_q4(cache.c, b, 1, out if dim else None, dq if dim else None, dk, dv, heads, stride, stride, kv_stride, rope)
    torch.cuda.synchronize()
    want = cache.reference()
    turned_k = ref.rotate(k, dtype, table, positions, dim, adjacent) if dim else k
    want.write(1, slots, turned_k, v)
    got = cache.bytes()
    same = got == want.bytes
    assert bool(same.all()), (dtype, d, np.argwhere(~same)[:5], got[~same][:5], want.bytes[~same][:5])
    if pad:
        assert bool((cache.store[:, cache.size:] == 0xA5).all())
    if dim:
        turned = ref.rotate(q, dtype, table, positions, dim, adjacent)
        assert np.array_equal(host16(out).reshape(n, heads, d), turned)
    # and back
    gk, gv = (torch.zeros(n, kv_heads, d, dtype=KIND[dtype], device="cuda") for _ in range(2))
    sg.sgmv_kv_read_q4(cache.c, 1, gk, gv, kv_heads * d, ints(slots), n)
    inside = (np.asarray(slots) >= 0) & (np.asarray(slots) < n_pages * page)
    for g, w in zip((gk, gv), want.rows(1, np.asarray(slots)[inside], fp32=True)):
        with np.errstate(over="ignore"):
            assert np.array_equal(decode64(host16(g)[inside], dtype), decode64(round16(w, dtype), dtype), equal_nan=True)
    return cache, want


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,heads,kv_heads,page,n,dim,adjacent", [
    (128, 32, 32, 16, 1, 128, 0), (128, 8, 2, 16, 37, 128, 0), (128, 3, 1, 64, 61, 64, 1), (128, 4, 4, 32, 9, 0, 0),
    (64, 7, 1, 16, 33, 64, 0), (64, 4, 2, 128, 130, 32, 1), (64, 5, 5, 256, 19, 16, 0), (128, 5, 5, 32, 20, 112, 0),
    (128, 40, 8, 16, 259, 128, 1), (64, 1, 1, 16, 5, 48, 1)])
def test_append_writes_the_bytes_of_the_definition(dtype, d, heads, kv_heads, page, n, dim, adjacent):
    append_case(dtype, d, heads, kv_heads, page, n, dim, adjacent, seed=n)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append_of_fused_rows_in_place_and_padded_pages(dtype):
    append_case(dtype, 128, 6, 2, 16, 45, 128, 0, seed=5, pad=48, fused=True)
    append_case(dtype, 64, 6, 3, 32, 45, 64, 1, seed=6, pad=16, fused=True)


def test_append_skips_slots_and_positions_out_of_range():
    slots = np.array([3, -1, 4, 16 * 5, 6, 1 << 30, 79, -(1 << 31)])
    append_case("f16", 128, 4, 2, 16, 8, 128, 0, slots=slots, special=False)  # 8 // 16 + 3 = 3 pages: 79 and 80 are outside too
    cache = Cache("f16", 128, 2, 1, 16, 3)
    rng = np.random.default_rng(0)
    q, k, v = (bits16(normal(rng, (4, 2, 128), "f16"), "f16") for _ in range(3))
    out = torch.full_like(q, 7.0)
    table = dev(rope_table(10, 128))
    slots, positions = ints([0, 1, 2, 3]), ints([9, 10, -1, 0])
    b = sg.make_kv_batch(1, 4, 1, None, None, None, slots, positions)
    sg.sgmv_kv_append_q4(cache.c, b, 0, out, q, k, v, 2, 256, 256, 256, sg.make_rope(table, 10, 128))
    out = host(out)
    assert (out[1:3] == 7.0).all() and (out[0] != 7.0).any() and (out[3] != 7.0).any()
    tile = cache.bytes()[0, 0, 0, 0]
    params = tile[2048:2048 + 16].reshape(4, 4)
    assert (params[1:3] == 0xA5).all() and (params[0] != 0xA5).any() and (params[3] != 0xA5).any()


# ---------------------------------------------------------------------------------------------- assign

def assign_case(page, n_pages, width, n_tokens, new, old, tables, stack, count, in_place=False, stream=None):
    c = sg.make_kv_cache(sg.F16, 128, 2, 1, page, n_pages)
    n = len(new)
    t, lens, out_lens = ints(tables), ints(old), ints(np.zeros(n))
    free, cnt, cnt_out = ints(stack), ints([count]), ints([-7])
    q_starts, slots, positions, status = ints(np.full(n + 1, -9)), ints(np.full(n_tokens, -9)), ints(np.full(n_tokens, -9)), ints([0, 64])
    if in_place:
        out_lens, cnt_out = lens, cnt
    b = sg.make_kv_batch(n, n_tokens, width, q_starts, out_lens, t, slots, positions)
    fresh = ints(new)
    sg.sgmv_kv_assign(c, b, fresh, lens, free, cnt, cnt_out, status, stream)
    torch.cuda.synchronize()
    want = ref.assign(page, n_pages, width, n_tokens, new, old, tables, stack, count)
    names = ("lens", "tables", "stack", "count", "q_starts", "slots", "positions")
    for name, g, w in zip(names, (out_lens, t, free, cnt_out, q_starts, slots, positions), want[1:]):
        assert np.array_equal(host(g).reshape(-1), np.asarray(w).reshape(-1)), (name, host(g), w)
    assert host(status).tolist() == [want[0], want[0] | 64]
    return want[0]


def random_step(rng, n, page, longest, tokens, over=0.2, spare=5):
    old = rng.integers(0, longest + 1, n)
    new = np.where(rng.random(n) < over, -1, rng.integers(0, tokens + 1, n))
    held = -(-old // page)
    later = -(-(old + np.maximum(new, 0)) // page)
    width = int(later.max()) + 1
    need = int((later - held).sum())
    n_pages = int(held.sum()) + need + spare
    ids = rng.permutation(n_pages)
    tables = np.full((n, width), -1)
    at = 0
    for i in range(n):
        tables[i, :held[i]] = ids[at:at + held[i]]
        at += held[i]
    stack = np.full(n_pages, -1)
    count = n_pages - at
    stack[:count] = ids[at:]
    return page, n_pages, width, new, old, tables, stack, count


@pytest.mark.parametrize("n,page,longest,tokens", [(1, 16, 0, 1), (1, 16, 40, 500), (3, 32, 100, 2), (64, 16, 300, 1), (65, 64, 300, 90),
                                                   (1023, 16, 60, 3), (1025, 16, 90, 2), (3000, 32, 500, 1), (130, 256, 1000, 200),
                                                   (4097, 16, 40, 1), (5000, 16, 20, 3), (9000, 32, 60, 2)])
@pytest.mark.parametrize("in_place", [False, True])
def test_assign(n, page, longest, tokens, in_place):
    rng = np.random.default_rng(n + page)
    page, n_pages, width, new, old, tables, stack, count = random_step(rng, n, page, longest, tokens)
    rows = int(np.maximum(new, 0).sum())
    for extra in (0, 1, 300):
        assert assign_case(page, n_pages, width, rows + extra, new, old, tables, stack, count, in_place) == 0


def test_assign_refuses_the_whole_step():
    rng = np.random.default_rng(4)
    for n in (5, 1500):
        page, n_pages, width, new, old, tables, stack, count = random_step(rng, n, 16, 100, 20, over=0.0)
        new[n // 2], old[n // 2] = 20, 7
        rows = int(new.sum())
        again = lambda **k: assign_case(*{**dict(page=page, n_pages=n_pages, width=width, n_tokens=rows + 40, new=new, old=old,  # noqa: E731
                                                 tables=tables, stack=stack, count=count), **k}.values())
        assert again(count=0) & 1
        assert again(count=n_pages + 1) == 8 and again(count=-1) == 8
        assert again(n_tokens=max(0, int(np.maximum(new, 0).sum()) - 1)) == 4
        long = new.copy()
        long[n - 1] = width * page + 1
        assert again(new=long) & 2
        for bad_new, bad_old in ((-2, 0), (0, -1), (0, width * page + 1)):
            a, o = new.copy(), old.copy()
            a[0], o[0] = bad_new, bad_old
            assert again(new=a, old=o) & 8
        # every length at its largest: sums pass 32 bits
        assert again(new=np.full(n, 2**31 - 1)) & 2


def test_assign_takes_a_page_that_is_not_of_the_cache_for_absent():
    tables = np.array([[0, -1], [1, -1]])
    stack = np.array([2, 99, -1, -1])
    assert assign_case(16, 4, 2, 5, [2, 1], [16, 3], tables, stack, 2) == 16


def test_assign_step_after_step_in_a_graph():
    """A captured decode step, replayed: pages come from the stack as the lengths pass page borders, and the host does nothing."""
    n, page, width, n_pages = 5, 16, 8, 40
    c = sg.make_kv_cache(sg.F16, 128, 2, 1, page, n_pages)
    lens, count = ints([0, 15, 16, 31, 1]), ints([n_pages - 6])
    tables = np.full((n, width), -1)
    for i, own in enumerate(([], [0], [1], [2, 3], [4])):
        tables[i, :len(own)] = own
    order = np.r_[np.arange(5, n_pages - 1), np.full(6, -1)]
    t, stack, new = ints(tables), ints(order), ints(np.ones(n))
    q_starts, slots, positions, status = ints(np.zeros(n + 1)), ints(np.zeros(n)), ints(np.zeros(n)), ints([0, 0])
    b = sg.make_kv_batch(n, n, width, q_starts, lens, t, slots, positions)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            sg.sgmv_kv_assign(c, b, new, lens, stack, count, count, status, stream)
        stream.synchronize()
        hl, hc, ht, hs = np.array([0, 15, 16, 31, 1]), n_pages - 6, tables, order
        for _ in range(40):
            g.replay()
            torch.ones(100, device="cuda").sum().item()
            stream.synchronize()
            _, hl, ht, hs, hc, _, want_slots, want_positions = ref.assign(page, n_pages, width, n, np.ones(n, int), hl, ht, hs, hc)
            assert host(lens).tolist() == list(hl) and host(count).tolist() == [hc]
            assert np.array_equal(host(slots), want_slots) and np.array_equal(host(positions), want_positions)
    assert host(status).tolist() == [0, 0]


# ---------------------------------------------------------------------------------------------- attention

def filled_cache(rng, dtype, d, kv_heads, page, lens, layers=2, spare=2, width_more=1, fill=0xFF, q_scale=1.0):
    """A cache whose layer 1 holds rows of every request, everything else a pattern whose scales are NaN."""
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + spare
    width = max(held) + width_more
    ids = rng.permutation(n_pages)
    tables = np.full((len(lens), width), 1 << 30)
    at = 0
    for i, h in enumerate(held):
        tables[i, :h] = ids[at:at + h]
        at += h
    cache = Cache(dtype, d, kv_heads, layers, page, n_pages, fill=fill)
    pages = cache.reference(fill)
    for i, n in enumerate(lens):
        if n:
            p = np.arange(n)
            pages.write(1, tables[i, p // page] * page + p % page, normal(rng, (n, kv_heads, d), dtype), normal(rng, (n, kv_heads, d), dtype, 0.3))
    cache.put(pages)
    return cache, pages, tables


def rows_of(pages, tables, page, bad=()):
    def of(r, positions):
        slots = tables[r, positions // page] * page + positions % page
        slots = np.where((tables[r, positions // page] < 0) | (tables[r, positions // page] >= pages.bytes.shape[0]), 0, slots)
        return pages.rows(1, slots)
    return of


def attend(cache, tables, starts, lens, q, heads, scale, causal=1, window=0, scratch=0, lse=True, hints=(0, 0), out_pad=0, n_tokens=None,
           stream=None, out=None):
    n = n_tokens if n_tokens is not None else q.shape[0]
    d = cache.d
    q_starts, kv_lens, t = ints(starts), ints(lens), ints(tables)
    b = sg.make_kv_batch(len(lens), n, tables.shape[1], q_starts, kv_lens, t, max_q_len=hints[0], max_kv_len=hints[1])
    if out is None:
        out = torch.full((n, heads * d + out_pad), -3.0, dtype=KIND[cache.dtype], device="cuda")
    sums = torch.full((n, heads), -3.0, device="cuda") if lse else None
    work = torch.full((scratch,), 0xFF, dtype=torch.uint8, device="cuda") if scratch else None
    sg.sgmv_attention_q4(cache.c, b, 1, out, sums, q, heads, out.shape[1], q.stride(0), scale, causal, window, work, scratch, stream)
    torch.cuda.synchronize()
    return out, sums


def check_attention(dtype, d, heads, kv_heads, page, lens, new, causal=1, window=0, scratch=0, seed=0, scale=None, hints=(0, 0), tail=2, q_size=1.0):
    rng = np.random.default_rng(seed)
    cache, pages, tables = filled_cache(rng, dtype, d, kv_heads, page, lens)
    starts = np.concatenate(([0], np.cumsum(new)))
    t = int(starts[-1])
    q = normal(rng, (t + tail, heads, d), dtype, q_size)
    scale = d ** -0.5 if scale is None else scale
    dq = bits16(q.reshape(t + tail, heads * d), dtype)
    out, lse = attend(cache, tables, starts, lens, dq, heads, scale, causal, window, scratch, hints=hints, out_pad=8)
    got = decode64(host16(out[:, :heads * d]), dtype).reshape(t + tail, heads, d)
    assert (host(out[:, heads * d:].float()) == -3).all() and (got[t:] == -3).all() and (host(lse)[t:] == -3).all()
    want, want_lse, off, spread = ref.attention(decode64(q, dtype)[:t], rows_of(pages, tables, page), starts, lens, heads, kv_heads, scale, causal, window)
    error = np.abs(got[:t] - want)
    bound = ref.tolerance(want, off, spread, dtype)
    assert (error <= bound).all(), (np.argwhere(error > bound)[:4], error.max(), (error / bound).max())
    if np.linalg.norm(want) > 0:
        # of the whole, a rounding is off by less than its largest, and everything before it by less than half of that
        assert np.linalg.norm(got[:t] - want) <= 1.5 * ref.HALF_STEP[dtype] * np.linalg.norm(want)
    gl = host(lse)[:t].astype(np.float64)
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(gl), empty) and (got[:t][empty] == 0).all()
    assert (np.abs(gl - np.where(empty, 0, want_lse))[~empty] <= (off + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, want_lse))))[~empty]).all()
    return out


SHAPES = [(128, 2, 2), (128, 8, 2), (128, 7, 1), (64, 4, 4), (64, 14, 2), (128, 20, 1), (64, 33, 1)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,heads,kv_heads", SHAPES)
def test_attention_single_tokens(dtype, d, heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 129, 300, 0]
    check_attention(dtype, d, heads, kv_heads, 16, lens, [1] * len(lens), seed=heads)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,heads,kv_heads", SHAPES)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_attention_rows_of_prompts_and_single_tokens(dtype, d, heads, kv_heads, page):
    lens, new = [40, 7, 133, 0, 90, 17, 65], [40, 7, 1, 0, 33, 2, 0]
    check_attention(dtype, d, heads, kv_heads, page, lens, new, seed=page)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [1, 3, 16, 33, 1000])
@pytest.mark.parametrize("causal", [0, 1])
def test_attention_windows_and_all_positions(dtype, window, causal):
    check_attention(dtype, 128, 6, 2, 32, [1, 90, 130, 64], [1, 37, 1, 64], causal, window, seed=window)
    check_attention(dtype, 64, 3, 3, 16, [50, 200], [50, 3], causal, window, seed=window)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
def test_attention_more_rows_than_positions(dtype, causal):
    """The first rows stand before position 0: with a causal mask they see nothing."""
    check_attention(dtype, 128, 4, 2, 16, [3, 0, 20], [9, 4, 36], causal, seed=1)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,heads,kv_heads", [(128, 4, 4), (64, 7, 1), (128, 16, 2)])
@pytest.mark.parametrize("hints", [(0, 0), (1, 100), (1, 5000), (700, 1)])
def test_attention_in_slices(dtype, d, heads, kv_heads, hints):
    """With a workspace long contexts are divided, with wrong hints too; ragged ones leave slices empty."""
    lens, new = [1000, 1, 260, 0, 777, 31], [1, 1, 3, 1, 1, 0]
    a = check_attention(dtype, d, heads, kv_heads, 16, lens, new, scratch=1 << 24, hints=hints, seed=3)
    b = check_attention(dtype, d, heads, kv_heads, 16, lens, new, scratch=1 << 24, hints=hints, seed=3)
    assert torch.equal(a, b)
    check_attention(dtype, d, heads, kv_heads, 16, lens, new, 1, 200, scratch=1 << 24, hints=hints, seed=3)


def plan_of(cache, lens, new, heads, hints, scratch=0, window=0, width=None):
    width = width or max(-(-n // cache.page) for n in lens) + 1
    b = sg.make_kv_batch(len(lens), sum(new), width, None, None, None, max_q_len=hints[0], max_kv_len=hints[1])
    return sg.sgmv_plan_attention_q4(cache.c, b, heads, window, 1 << 8 if scratch else None, scratch)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kv_heads,group,hints,actual", [(5, 1, (1, 40), 1), (5, 2, (1, 600), 1), (6, 3, (5, 40), 5), (5, 3, (1, 30), 9), (7, 17, (0, 0), 1)])
def test_attention_of_many_short_requests(dtype, kv_heads, group, hints, actual):
    """More requests than a wave orders at once; a wave to a head (and heads that do not fill the last workgroup); more rows and positions
    than the hint says."""
    rng = np.random.default_rng(kv_heads + group)
    n = 330
    lens = rng.integers(0, 45, n)
    lens[7], lens[200] = 300, 0
    new = np.minimum(rng.integers(0, actual + 1, n), lens + 1)
    cache = Cache(dtype, 64, kv_heads, 1, 16, 4)
    plan = plan_of(cache, lens.tolist(), new.tolist(), kv_heads * group, hints)
    if hints[0] * group in range(1, 17):
        assert plan.kernel == sg.KERNEL_ATTENTION_FEW
        assert plan.workgroups == (n * -(-kv_heads // 4) if hints[1] <= 640 else n * kv_heads)
    check_attention(dtype, 64, kv_heads * group, kv_heads, 16, lens.tolist(), new.tolist(), hints=hints, seed=n)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,kv_heads,group", [(128, 24, 1), (64, 24, 2), (128, 7, 5)])
@pytest.mark.parametrize("hint", [0, 130])
def test_attention_tiles_of_many_prompts(dtype, d, kv_heads, group, hint):
    """Prompts and single tokens in tiles ordered by their work: whole tiles, ends of 1 to 127 columns (waves that share them), requests without
    rows, more than 128 tiles."""
    lens = [130, 1, 33, 64, 0, 17, 100, 40, 65, 3, 129, 48, 31, 96, 20, 77]
    new = [130, 1, 33, 1, 0, 16, 100, 0, 65, 2, 1, 48, 31, 90, 20, 13]
    check_attention(dtype, d, kv_heads * group, kv_heads, 16, lens, new, hints=(hint, hint), seed=kv_heads)
    if kv_heads == 7:
        check_attention(dtype, d, kv_heads * group, kv_heads, 32, lens * 9, new * 9, hints=(hint, hint), window=50, seed=1)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("requests,kv_heads,group,columns", [(1, 3, 2, 16), (8, 64, 1, 32), (8, 64, 2, 64), (8, 64, 5, 128)])
def test_attention_tiles_of_every_width(dtype, d, requests, kv_heads, group, columns):
    lens, new = [20 + 3 * (i % 5) for i in range(requests)], [20] * requests
    cache = Cache(dtype, d, kv_heads, 1, 16, 4)
    plan = plan_of(cache, lens, new, kv_heads * group, (20, max(lens)))
    assert plan.kernel == sg.KERNEL_ATTENTION_MANY and plan.workgroups == (20 * requests * group // columns + requests) * kv_heads
    check_attention(dtype, d, kv_heads * group, kv_heads, 16, lens, new, hints=(20, max(lens)), seed=columns)
    check_attention(dtype, d, kv_heads * group, kv_heads, 16, lens, [20, 1, 0, 13, 20, 7, 20, 2][:requests], window=9, hints=(20, max(lens)), seed=columns)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("hints", [(40, 700), (40, 100000), (1000, 0)])
def test_attention_of_prompts_in_slices(dtype, hints):
    """Rows behind long contexts, in slices; rows whose positions fit one slice are written by it, those without any by the join or not at all."""
    lens, new = [700, 40, 0, 333, 20, 64], [40, 40, 1, 1, 0, 64]
    for window in (0, 300):
        check_attention(dtype, 128, 10, 2, 16, lens, new, 1, window, scratch=1 << 25, hints=hints, seed=5)
    check_attention(dtype, 64, 4, 4, 16, lens, new, 0, 0, scratch=1 << 25, hints=hints, seed=6)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_of_sharp_and_flat_softmaxes(dtype):
    for q_size, scale in ((30.0, 0.3), (1e-3, 1e-3), (0.0, 1.0), (1.0, 1e-30), (100.0, 1.0)):
        check_attention(dtype, 128, 4, 2, 16, [100, 37], [5, 1], q_size=q_size, scale=scale, seed=9)


def test_attention_of_the_largest_and_smallest_bfloat16_rows():
    """Rows of q far outside binary16's range, up and down."""
    for size in (1e-36, 1e-20, 1e20, 1e28):
        check_attention("bf16", 128, 4, 2, 16, [100, 37], [5, 1], q_size=size, scale=0.1 / size, seed=9)


def test_attention_scales_of_v_far_apart():
    """Scales of v that grow by 2^40 along the positions, and back: the weights' unit follows, what is small next to it stays seen where it counts."""
    rng = np.random.default_rng(0)
    for order in (1, -1):
        lens = [300]
        cache, pages, tables = filled_cache(rng, "bf16", 128, 2, 16, lens)
        size = 2.0 ** np.linspace(-20, 20, 300)[::order]
        v = round16((rng.standard_normal((300, 2, 128)) * size[:, None, None]).astype(np.float32), "bf16")
        k = normal(rng, (300, 2, 128), "bf16")
        p = np.arange(300)
        pages.write(1, tables[0, p // 16] * 16 + p % 16, k, v)
        cache.put(pages)
        q = normal(rng, (300, 4, 128), "bf16")
        out, _ = attend(cache, tables, [0, 300], lens, bits16(q.reshape(300, -1), "bf16"), 4, 0.088)
        want, _, off, spread = ref.attention(decode64(q, "bf16"), rows_of(pages, tables, 16), [0, 300], lens, 4, 2, 0.088)
        got = decode64(host16(out), "bf16").reshape(300, 4, 128)
        # a row's own sum is held next to the largest scale that any row of its tile sees: 2^-36 of that, times a code
        slack = 2.0 ** -31 * np.abs(decode64(v, "bf16")).max()
        assert (np.abs(got - want) <= ref.tolerance(want, off, spread, "bf16") + slack).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_what_is_not_finite(dtype):
    """A row of q, a key or a value that is not finite makes NaN of what sees it, and of nothing else."""
    rng = np.random.default_rng(2)
    lens, new = [60, 60, 60, 60], [4, 4, 4, 4]
    cache, pages, tables = filled_cache(rng, dtype, 128, 2, 16, lens)
    starts = np.arange(0, 17, 4)
    slot = lambda r, p: tables[r, p // 16] * 16 + p % 16  # noqa: E731
    k, v = (normal(rng, (1, 2, 128), dtype) for _ in range(2))
    bad = k.copy()
    bad[0, 1, 5] = 0x7FFF
    pages.write(1, [slot(1, 58)], bad, v)   # rows 0 and 1 of request 1 stand at 56 and 57: they do not see it
    pages.write(1, [slot(2, 57)], k, bad)
    pages.write(1, [slot(3, 59)], bad, bad)
    cache.put(pages)
    q = normal(rng, (16, 4, 128), dtype)
    q[1, 2, 7] = 0x7FFF
    q[2, 0, 9] = 0xFF80 if dtype == "bf16" else 0xFC00
    out, lse = attend(cache, tables, starts, lens, bits16(q.reshape(16, -1), dtype), 4, 0.088)
    got = decode64(host16(out), dtype).reshape(16, 4, 128)
    nan = np.isnan(got)
    assert np.array_equal(nan.all(-1), nan.any(-1))
    want = np.zeros((16, 4), bool)
    want[1, 2] = want[2, 0] = True
    want[6:8, 2:] = want[9:12, 2:] = want[15, 2:] = True
    assert np.array_equal(nan.all(-1), want)
    clean, _, off, spread = ref.attention(decode64(np.where(want[..., None], 0, q), dtype), rows_of(pages, tables, 16), starts, lens, 4, 2, 0.088)
    fine = ~want
    assert (np.abs(got - clean)[fine] <= ref.tolerance(clean, off, spread, dtype)[fine]).all()


@pytest.mark.parametrize("fill", [0x00, 0x7B, 0x7F, 0xFF])
@pytest.mark.parametrize("window", [0, 20])
def test_attention_pages_that_are_absent_and_what_lies_around(fill, window):
    """Entries of a table outside the cache hide their positions; unwritten positions of a last page may hold anything (0x7B7B: the largest
    scales of binary16)."""
    rng = np.random.default_rng(7)
    lens, new = [70, 41, 100], [3, 1, 70]
    cache, pages, tables = filled_cache(rng, "f16", 128, 2, 16, lens, fill=fill)
    tables[0, 1], tables[2, 0], tables[2, 4] = -1, pages.bytes.shape[0], -(1 << 31)
    starts = np.concatenate(([0], np.cumsum(new)))
    q = normal(rng, (74, 4, 128), "f16")
    out, lse = attend(cache, tables, starts, lens, bits16(q.reshape(74, -1), "f16"), 4, 0.088, window=window)
    gone = lambda r: np.isin(np.arange(lens[r]) // 16, {0: [1], 1: [], 2: [0, 4]}[r])  # noqa: E731
    want, want_lse, off, spread = ref.attention(decode64(q, "f16"), rows_of(pages, tables, 16), starts, lens, 4, 2, 0.088, True, window, gone)
    got = decode64(host16(out), "f16").reshape(74, 4, 128)
    assert (np.abs(got - want) <= ref.tolerance(want, off, spread, "f16")).all()
    assert np.array_equal(np.isneginf(host(lse)), np.isneginf(want_lse))


def test_attention_takes_lengths_and_starts_that_lead_out_for_absent():
    rng = np.random.default_rng(8)
    lens = [40, 30]
    cache, pages, tables = filled_cache(rng, "f16", 64, 2, 16, lens, width_more=0)
    tables = np.where(tables >= pages.bytes.shape[0], -1, tables)
    q = normal(rng, (6, 2, 64), "f16")
    dq = bits16(q.reshape(6, -1), "f16")
    # a length past the table is cut to it, a negative one to nothing; the second request's rows end behind the batch
    out, _ = attend(cache, tables, [0, 2, 9], [1 << 30, -5], dq, 2, 0.1, causal=0)
    got = decode64(host16(out), "f16").reshape(6, 2, 64)
    # positions 40 .. 47 of the first request hold NaN scales
    assert np.isnan(got[:2]).all() and (got[2:] == 0).all()
    out, _ = attend(cache, tables, [0, 2, 9], [40, 30], dq, 2, 0.1, causal=0)
    want, *_ = ref.attention(decode64(q, "f16"), rows_of(pages, tables, 16), [0, 2, 6], [40, 30], 2, 2, 0.1, causal=False)
    assert np.abs(decode64(host16(out), "f16").reshape(6, 2, 64) - want).max() < 0.01
    for starts in ([-4, 3, 2], [5, 5, 5], [1 << 30, 0, 6], [6, 4, 2]):
        attend(cache, tables, starts, [40, 30], dq, 2, 0.1)  # nothing but: no access leaves a buffer


def test_attention_one_long_context():
    """131 072 positions less a few, shared heads: slices, and lookups far into a table."""
    rng = np.random.default_rng(11)
    n, d, page = 131071, 128, 64
    held = -(-n // page)
    cache = Cache("bf16", d, 2, 2, page, held + 1)
    tables = rng.permutation(held + 1)[None, :held]
    k, v = (torch.randn(n, 2, d, device="cuda", dtype=torch.float32).bfloat16() for _ in range(2))
    p = np.arange(n)
    slots = ints(tables[0, p // page] * page + p % page)
    b = sg.make_kv_batch(1, n, held, None, None, None, slots)
    sg.sgmv_kv_append_q4(cache.c, b, 1, None, None, k, v, 8, 8 * d, 8 * d, 2 * d)
    kq, vq = torch.zeros_like(k), torch.zeros_like(v)
    sg.sgmv_kv_read_q4(cache.c, 1, kq, vq, 2 * d, slots, n)
    q = torch.randn(2, 8 * d, device="cuda").bfloat16()
    for scratch in (0, 1 << 22, 1 << 26):
        out, lse = attend(cache, tables, [0, 2], [n], q, 8, d ** -0.5, scratch=scratch, hints=(2, n))
        x = torch.einsum("thd,phd->thp", q.view(2, 8, d).double(), kq.double().repeat_interleave(4, 1)) * d ** -0.5
        x[0, :, -1] = -np.inf
        want = torch.einsum("thp,phd->thd", torch.softmax(x, -1), vq.double().repeat_interleave(4, 1))
        # the rows read back are rounded to 16 bits, which the kernel's are not: half a step of a score's and a value's parts each
        assert float((out.view(2, 8, d).double() - want).norm() / want.norm()) < 3 * 2.0 ** -8
        assert float((lse.double() - torch.logsumexp(x, -1)).abs().max()) < 0.01


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_odd_positions_of_one_sign(dtype):
    """Values that are all large and of one sign next to a small spread, and all alike: the codes' sums nearly cancel against the minima."""
    rng = np.random.default_rng(21)
    lens = [513, 2]
    for size, spread in ((100.0, 1.0), (1.0, 0.0), (-50.0, 0.25)):
        cache, pages, tables = filled_cache(rng, dtype, 128, 1, 16, lens)
        for r, n in enumerate(lens):
            p = np.arange(n)
            v = round16((size + spread * rng.standard_normal((n, 1, 128))).astype(np.float32), dtype)
            pages.write(1, tables[r, p // 16] * 16 + p % 16, normal(rng, (n, 1, 128), dtype), v)
        cache.put(pages)
        q = normal(rng, (5, 3, 128), dtype)
        out, _ = attend(cache, tables, [0, 3, 5], lens, bits16(q.reshape(5, -1), dtype), 3, 0.05, scratch=1 << 22)
        want, _, off, weighed = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), [0, 3, 5], lens, 3, 1, 0.05)
        assert (np.abs(decode64(host16(out), dtype).reshape(5, 3, 128) - want) <= ref.tolerance(want, off, weighed, dtype)).all()


@pytest.mark.parametrize("dtype,value,lens", [("f16", 40000.0, [9000, 33]), ("f16", -65504.0, [8200]), ("bf16", 1e9, [513]), ("bf16", -1e30, [513, 40]),
                                              ("bf16", 2e38, [300]), ("bf16", 0.0, [513, 1]), ("f16", 0.0, [40])])
def test_attention_constant_values(dtype, value, lens):
    """Rows of v without a scale: nothing but minima, up to the type's largest."""
    rng = np.random.default_rng(7)
    cache, pages, tables = filled_cache(rng, dtype, 64, 1, 16, lens)
    value = decode64(round16(np.full(1, value, np.float32), dtype), dtype)[0]
    for r, n in enumerate(lens):
        p = np.arange(n)
        pages.write(1, tables[r, p // 16] * 16 + p % 16, normal(rng, (n, 1, 64), dtype), round16(np.full((n, 1, 64), value, np.float32), dtype))
    cache.put(pages)
    new = [1] * len(lens)
    starts = np.concatenate(([0], np.cumsum(new)))
    q = normal(rng, (len(lens), 4, 64), dtype)
    for scratch in (0, 1 << 22):
        out, lse = attend(cache, tables, starts, lens, bits16(q.reshape(len(lens), -1), dtype), 4, 0.125, scratch=scratch)
        want, want_lse, off, _ = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), starts, lens, 4, 1, 0.125)
        got = decode64(host16(out), dtype).reshape(want.shape)
        # the same weights in the sum and under it, n additions of fp32 each
        assert (np.abs(got - value) <= abs(value) * (ref.HALF_STEP[dtype] + 2.0 ** -24 * (2 * max(lens) + 16))).all()
        assert (np.abs(host(lse).astype(np.float64) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("scratch", [0, 1 << 20])
def test_attention_tiny_scores_and_a_hidden_page(scratch):
    """Scores so small that their factor is no number of fp32, next to a page that is not of the cache: all weights alike, its own nothing."""
    rng = np.random.default_rng(8)
    lens = [256]
    cache, pages, tables = filled_cache(rng, "bf16", 128, 1, 16, lens)
    tables[0, 3] = -1
    q = normal(rng, (1, 2, 128), "bf16", 1e-36)
    out, lse = attend(cache, tables, [0, 1], lens, bits16(q.reshape(1, -1), "bf16"), 2, 1e-20, scratch=scratch)
    hidden = lambda r: np.arange(256) // 16 == 3
    want, want_lse, off, spread = ref.attention(decode64(q, "bf16"), rows_of(pages, tables, 16), [0, 1], lens, 2, 1, 1e-20, hidden=hidden)
    assert (np.abs(decode64(host16(out), "bf16").reshape(want.shape) - want) <= ref.tolerance(want, off, spread, "bf16")).all()
    assert (np.abs(host(lse) - want_lse) <= 1e-5).all()


def test_attention_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(12)
    lens, new = [300, 40, 17], [1, 5, 1]
    cache, pages, tables = filled_cache(rng, "f16", 128, 2, 16, lens)
    starts = [0, 1, 6, 7]
    q = bits16(normal(rng, (7, 1024), "f16"), "f16")
    eager, _ = attend(cache, tables, starts, lens, q, 8, 0.088, scratch=1 << 20, lse=False)
    q_starts, kv_lens, t = ints(starts), ints(lens), ints(tables)
    b = sg.make_kv_batch(3, 7, tables.shape[1], q_starts, kv_lens, t)
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    out = torch.zeros(7, 1024, dtype=torch.float16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    sg.sgmv_attention_q4(cache.c, b, 1, out, None, q, 8, 1024, 1024, 0.088, 1, 0, scratch, 1 << 20, stream)
    stream.synchronize()
    assert torch.equal(out, eager)
    other = torch.zeros_like(out)
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            # two calls share the workspace, one after the other
            sg.sgmv_attention_q4(cache.c, b, 1, out, None, q, 8, 1024, 1024, 0.088, 1, 0, scratch, 1 << 20, stream)
            sg.sgmv_attention_q4(cache.c, b, 1, other, None, q, 8, 1024, 1024, 0.5, 1, 0, scratch, 1 << 20, stream)
    sharp, _ = attend(cache, tables, starts, lens, q, 8, 0.5, scratch=1 << 20, lse=False)
    for i in range(4):
        out.zero_(), other.zero_(), scratch.fill_(0xFF)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(other, sharp), i


def test_two_calls_at_once_on_streams_of_their_own():
    """The same cache and batch, workspaces apart."""
    rng = np.random.default_rng(14)
    lens = [3000, 2500]
    cache, pages, tables = filled_cache(rng, "bf16", 128, 2, 16, lens)
    q = bits16(normal(rng, (2, 1024), "bf16"), "bf16")
    scales = (0.05, 0.2)
    want = [attend(cache, tables, [0, 1, 2], lens, q, 8, s, scratch=1 << 20, hints=(1, 3000), lse=False)[0] for s in scales]
    q_starts, kv_lens, t = ints([0, 1, 2]), ints(lens), ints(tables)
    b = sg.make_kv_batch(2, 2, tables.shape[1], q_starts, kv_lens, t, max_q_len=1, max_kv_len=3000)
    assert sg.sgmv_plan_attention_q4(cache.c, b, 8, 0, 1 << 8, 1 << 20).slices > 1
    streams, works, outs = ([f() for _ in scales] for f in (torch.cuda.Stream, lambda: torch.empty(1 << 20, dtype=torch.uint8, device="cuda"),
                                                           lambda: torch.zeros(2, 1024, dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, work, out, scale in zip(streams, works, outs, scales):
            sg.sgmv_attention_q4(cache.c, b, 1, out, None, q, 8, 1024, 1024, scale, 1, 0, work, 1 << 20, stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_pages_far_apart():
    """A cache whose pages lie 2^30 bytes from one another: what it holds and gives is what a dense one does."""
    rng = np.random.default_rng(15)
    n_pages, page, d, stride = 6, 16, 64, 1 << 30
    store = torch.empty((n_pages - 1) * stride + (1 << 20), dtype=torch.uint8, device="cuda")
    far = sg.make_kv_cache(sg.F16, d, 2, 3, page, n_pages, store, stride)
    dense = Cache("f16", d, 2, 3, page, n_pages)
    n, new = 90, 20
    tables = np.array([[5, 0, 4, 1, 3, 2]])
    p = np.arange(n)
    slots, starts, lens, t = ints(tables[0, p // page] * page + p % page), ints([0, new]), ints([n]), ints(tables)
    k, v = (bits16(normal(rng, (n, 2 * d), "f16"), "f16") for _ in range(2))
    q = bits16(normal(rng, (new, 4 * d), "f16"), "f16")
    rows, results = sg.make_kv_batch(1, n, 6, None, None, None, slots), []
    for c in (far, dense.c):
        sg.sgmv_kv_append_q4(c, rows, 2, None, None, k, v, 4, 4 * d, 4 * d, 2 * d)
        out, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        sg.sgmv_attention_q4(c, sg.make_kv_batch(1, new, 6, starts, lens, t), 2, out, None, q, 4, 4 * d, 4 * d, 0.125)
        sg.sgmv_kv_read_q4(c, 2, gk, gv, 2 * d, slots, n)
        torch.cuda.synchronize()
        results.append((out, gk, gv))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and bool(results[0][0].abs().sum() > 0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("hint", [1, 30])
def test_attention_of_seventy_thousand_requests(dtype, hint):
    """A position each, so that every result is its row of v; every third request has no row."""
    n, d, heads = 70001, 64, 2
    cache = Cache(dtype, d, 1, 2, 16, n)
    tables = torch.randperm(n, device="cuda", dtype=torch.int32)[:, None].contiguous()
    slots = (tables[:, 0] * 16).contiguous()
    k, v = (torch.randn(n, d, device="cuda").to(KIND[dtype]) for _ in range(2))
    sg.sgmv_kv_append_q4(cache.c, sg.make_kv_batch(n, n, 1, None, None, None, slots), 1, None, None, k, v, heads, heads * d, heads * d, d)
    held = torch.zeros_like(v)
    sg.sgmv_kv_read_q4(cache.c, 1, None, held, d, slots, n)
    has = torch.arange(n, device="cuda") % 3 != 2
    starts = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), has.cumsum(0))).int()
    rows = int(starts[-1])
    q = torch.randn(rows, heads * d, device="cuda").to(KIND[dtype])
    out = torch.zeros_like(q)
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    b = sg.make_kv_batch(n, rows, 1, starts, lens, tables, max_q_len=hint, max_kv_len=1)
    assert sg.sgmv_plan_attention_q4(cache.c, b, heads).kernel == (sg.KERNEL_ATTENTION_FEW if hint == 1 else sg.KERNEL_ATTENTION_MANY)
    sg.sgmv_attention_q4(cache.c, b, 1, out, None, q, heads, heads * d, heads * d, 0.125)
    want = held[has][:, None].double()
    # the row is rounded once there, and here once after products and sums of fp32 (of the code, weighted, and the minimum: 2^-11 of the larger
    # part in bfloat16, whose weights have 11 bits)
    off = (out.view(rows, heads, d).double() - want).abs()
    spread = held[has].double().abs().amax(-1)[:, None, None]
    assert bool((off <= 2 * ref.HALF_STEP[dtype] * want.abs() + spread * (4 * ref.WEIGHT_STEP[dtype] + 2.0 ** -20)).all())


def test_a_served_batch_step_after_step():
    """assign, append and attend together: two prompts, then single tokens, one request over and another in its place."""
    rng = np.random.default_rng(13)
    dtype, d, heads, kv_heads, page, width, n_pages = "f16", 128, 4, 2, 16, 6, 14
    cache = Cache(dtype, d, kv_heads, 2, page, n_pages)
    table = rope_table(width * page, d)
    rope_dev = dev(table)
    rope = sg.make_rope(rope_dev, width * page, d)
    n, rows = 3, 64
    lens, count, stack, tables = ints(np.zeros(n)), ints([n_pages]), ints(np.arange(n_pages)), ints(np.full((n, width), -1))
    q_starts, slots, positions, status = ints(np.zeros(n + 1)), ints(np.zeros(rows)), ints(np.zeros(rows)), ints([0, 0])
    b = sg.make_kv_batch(n, rows, width, q_starts, lens, tables, slots, positions)
    q, k, v = (torch.zeros(rows, h * d, dtype=torch.float16, device="cuda") for h in (heads, kv_heads, kv_heads))
    turned, out = torch.zeros_like(q), torch.zeros_like(q)
    held_k, held_v = [[] for _ in range(n)], [[] for _ in range(n)]
    for step, new in enumerate([[37, 20, 0], [1, 1, 0], [1, 1, 5], [1, -1, 1], [1, 30, 1], [4, 1, 2], [-1, 1, 1], [1, 1, 1]]):
        hq, hk, hv = (normal(rng, (rows, h, d), dtype) for h in (heads, kv_heads, kv_heads))
        for t, x in ((q, hq), (k, hk), (v, hv)):
            t.copy_(bits16(x.reshape(rows, -1), dtype))
        out.fill_(-3.0)
        sg.sgmv_kv_assign(cache.c, b, ints(new), lens, stack, count, count, status)
        sg.sgmv_kv_append_q4(cache.c, b, 1, turned, q, k, v, heads, heads * d, heads * d, kv_heads * d, rope)
        sg.sgmv_attention_q4(cache.c, b, 1, out, None, turned, heads, heads * d, heads * d, d ** -0.5)
        torch.cuda.synchronize()
        starts, at = [0], np.zeros(rows, int)
        for r, a in enumerate(new):
            if a < 0:
                held_k[r], held_v[r] = [], []
            for j in range(max(a, 0)):
                at[starts[-1] + j] = len(held_k[r]) + j
            starts.append(starts[-1] + max(a, 0))
        t = starts[-1]
        tq, tk = (ref.rotate(x[:t], dtype, table, at[:t], d, 0) for x in (hq, hk))
        for r, a in enumerate(new):
            for j in range(starts[r], starts[r + 1]):
                held_k[r].append(tk[j]), held_v[r].append(hv[j])
        total = [len(x) for x in held_k]
        assert host(status).tolist() == [0, 0] and host(lens).tolist() == total and host(q_starts).tolist() == starts

        def of(r, positions):
            both = []
            for x in (held_k[r], held_v[r]):
                codes, s, m = ref.quantize(np.array(x), dtype)
                both.append(codes * decode64(s, dtype)[..., None] + decode64(m, dtype)[..., None])
            return both
        want, _, off, spread = ref.attention(decode64(tq, dtype), of, starts, total, heads, kv_heads, d ** -0.5)
        got = decode64(host16(out), dtype).reshape(rows, heads, d)
        assert (np.abs(got[:t] - want) <= ref.tolerance(want, off, spread, dtype)).all(), step
        assert (got[t:] == -3).all()

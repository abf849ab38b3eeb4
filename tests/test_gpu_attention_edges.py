"""Attention over the paged 4-bit cache where a column has seen nothing yet, sees nothing at all, or sees what lies far apart."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2310_18547_amd as sg
from backbone_reference import round16
from helpers import decode64
from test_gpu_attention import Cache, attend, bits16, check_attention, filled_cache, host, host16, normal, rows_of

pytestmark = pytest.mark.gpu


def slices_of(cache, tables, n_tokens, heads, hints, scratch, window=0):
    b = sg.make_kv_batch(len(tables), n_tokens, tables.shape[1], None, None, None, max_q_len=hints[0], max_kv_len=hints[1])
    return sg.sgmv_plan_attention_q4(cache.c, b, heads, window, 1 << 8 if scratch else None, scratch).slices


def plan_slices(dtype, d, heads, kv_heads, page, lens, new, hints, scratch, window=0, tail=2):
    """Slices of check_attention's call of these shapes."""
    held = [-(-n // page) for n in lens]
    c = sg.make_kv_cache(sg.F16 if dtype == "f16" else sg.BF16, d, kv_heads, 2, page, sum(held) + 2)
    b = sg.make_kv_batch(len(lens), sum(new) + tail, max(held) + 1, None, None, None, max_q_len=hints[0], max_kv_len=hints[1])
    return sg.sgmv_plan_attention_q4(c, b, heads, window, 1 << 8 if scratch else None, scratch).slices


# ---------------------------------------------------------------------------------------------- columns that have seen nothing yet

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,new", [(2, 2, 4), (4, 2, 4), (3, 1, 40)])
@pytest.mark.parametrize("window", [0, 150])
def test_zero_queries_whose_wave_begins_with_a_step_that_they_do_not_see(dtype, heads, kv_heads, new, window):
    """A wave takes the step that a mask cuts first, and its first rows see nothing there: their first score must still count, with scores of 0
    and a scale so small that the distance by which a maximum may lag is not finite."""
    for scale in (1 / 128, 1 / 512, 1e-30):
        check_attention(dtype, 128, heads, kv_heads, 16, [194], [new], window=window, q_size=0.0, scale=scale, seed=1)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [0, 3000])
def test_zero_queries_in_slices(dtype, window):
    for lens in ([4002], [4097], [4030]):
        hints, scratch = (4, lens[0]), 1 << 22
        assert plan_slices(dtype, 128, 2, 2, 16, lens, [4], hints, scratch, window) > 1
        check_attention(dtype, 128, 2, 2, 16, lens, [4], window=window, q_size=0.0, scale=1 / 128, scratch=scratch, hints=hints, seed=2)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,new", [(2, 4), (6, 30)])
@pytest.mark.parametrize("gone", [(0, 1), (2, 3, 4, 5), (0, 1, 4, 5, 8)])
def test_hidden_pages_behind_a_step_that_a_row_does_not_see(dtype, heads, new, gone):
    """The first step that a column sees whole lies on pages that are not of the cache, after its neighbours have raised their maxima."""
    rng = np.random.default_rng(len(gone))
    for n in (130, 131, 162):
        cache, pages, tables = filled_cache(rng, dtype, 128, 2, 16, [n])
        tables[0, list(gone)] = -1
        q = normal(rng, (new, heads, 128), dtype)
        out, lse = attend(cache, tables, [0, new], [n], bits16(q.reshape(new, -1), dtype), heads, 0.088)
        hidden = lambda r: np.isin(np.arange(n) // 16, gone)  # noqa: E731
        want, want_lse, off, spread = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), [0, new], [n], heads, 2, 0.088, hidden=hidden)
        got = decode64(host16(out), dtype).reshape(want.shape)
        assert (np.abs(got - want) <= ref.tolerance(want, off, spread, dtype)).all(), n
        assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


# ---------------------------------------------------------------------------------------------- rows that see nothing

@pytest.mark.parametrize("dtype,bad", [("f16", 0x7FFF), ("f16", 0x7C00), ("bf16", 0x7FFF), ("bf16", 0x7F80), ("bf16", 0x7200)])  # the last: 2^101
@pytest.mark.parametrize("heads", [2, 6])
@pytest.mark.parametrize("hints", [(0, 0), (2, 0)])
def test_queries_that_are_not_finite_and_see_nothing(dtype, bad, heads, hints):
    """Rows in front of position 0 are zeros with a sum of nothing, whatever they hold and whoever shares their tile."""
    rng = np.random.default_rng(3)
    lens, new = [3, 0, 40], [9, 4, 42]
    cache, pages, tables = filled_cache(rng, dtype, 128, 2, 16, lens)
    starts = np.concatenate(([0], np.cumsum(new)))
    q = normal(rng, (55, heads, 128), dtype)
    rows = [1, 7, 10, 14, 30]  # of the first request one in front of position 0 and one that sees positions, of the second, of the third as the first
    for row in rows:
        q[row, :, 5] = bad
    out, lse = attend(cache, tables, starts, lens, bits16(q.reshape(55, -1), dtype), heads, 0.088, hints=hints)
    got, sums = decode64(host16(out), dtype).reshape(55, heads, 128), host(lse)
    blind = np.r_[0:6, 9:13, 13:15]
    assert (got[blind] == 0).all() and np.isneginf(sums[blind]).all()
    for row in (7, 30):
        assert np.isnan(got[row]).all() and np.isnan(sums[row]).all()
    clean = q.copy()
    clean[rows] = 0
    want, want_lse, off, spread = ref.attention(decode64(clean, dtype), rows_of(pages, tables, 16), starts, lens, heads, 2, 0.088)
    fine = np.setdiff1d(np.arange(55), (7, 30))
    assert (np.abs(got - want)[fine] <= ref.tolerance(want, off, spread, dtype)[fine]).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [20, 32, 40, 300, 4000])
def test_queries_that_are_not_finite_over_hidden_pages(dtype, n):
    """NaN where positions are theirs to see, on pages of the cache or not; the others see nothing."""
    rng = np.random.default_rng(4)
    cache, pages, tables = filled_cache(rng, dtype, 64, 1, 16, [n])
    tables[:] = -1
    q = normal(rng, (3, 2, 64), dtype)
    q[1, 0, 3] = 0x7FFF
    hints, scratch = (3, n), 1 << 22
    assert n < 4000 or slices_of(cache, tables, 3, 2, hints, scratch) > 1
    for causal in (0, 1):
        out, lse = attend(cache, tables, [0, 3], [n], bits16(q.reshape(3, -1), dtype), 2, 0.125, causal, scratch=scratch, hints=hints)
        got, sums = decode64(host16(out), dtype).reshape(3, 2, 64), host(lse)
        bad = np.zeros((3, 2), bool)
        bad[1, 0] = True
        assert np.isnan(got[bad]).all() and np.isnan(sums[bad]).all()
        assert (got[~bad] == 0).all() and np.isneginf(sums[~bad]).all()


# ---------------------------------------------------------------------------------------------- scores and values far apart

FAR = [("f16", 200.0, 200.0, 0.088), ("f16", 3000.0, 3000.0, 0.088), ("f16", 3e4, 3e4, 0.088), ("bf16", 300.0, 1000.0, 0.088), ("bf16", 1e5, 1e5, 0.088),
       ("bf16", 2.0 ** 40, 2.0 ** 40, 1.0), ("bf16", 2.0 ** 50, 2.0 ** 49, 1.0), ("bf16", 2.0 ** -60, 2.0 ** -40, 2.0 ** 126)]


def far_case(rng, dtype, size, n, keys):
    """A cache of ``n`` positions whose keys are those of ``keys(k)``, made from one row of +-size and values of its own."""
    cache, pages, tables = filled_cache(rng, dtype, 128, 1, 16, [n])
    row = round16((size * rng.choice((-1.0, 1.0), 128)).astype(np.float32), dtype)
    k = keys(np.broadcast_to(row, (n, 1, 128)).copy())
    p = np.arange(n)
    pages.write(1, tables[0, p // 16] * 16 + p % 16, k, normal(rng, (n, 1, 128), dtype))
    cache.put(pages)
    return cache, pages, tables, row


@pytest.mark.parametrize("dtype,q_size,k_size,scale", FAR)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("n,scratch", [(20, 0), (300, 0), (2500, 1 << 22)])
def test_large_scores_that_are_all_alike(dtype, q_size, k_size, scale, sign, n, scratch):
    """Equal keys: every position weighs the same, however large the score (up to 2^107 here)."""
    rng = np.random.default_rng(5)
    cache, pages, tables, row = far_case(rng, dtype, k_size, n, lambda k: k)
    q = round16(np.broadcast_to((sign * q_size * np.sign(decode64(row, dtype))).astype(np.float32), (1, 2, 128)), dtype)
    hints = (1, n)
    assert not scratch or slices_of(cache, tables, 1, 2, hints, scratch) > 1
    out, lse = attend(cache, tables, [0, 1], [n], bits16(q.reshape(1, -1), dtype), 2, scale, scratch=scratch, hints=hints)
    want, want_lse, off, spread = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), [0, 1], [n], 2, 1, scale)
    assert np.abs(want_lse).max() > 100
    got = decode64(host16(out), dtype).reshape(want.shape)
    # scores of the same bytes are the same to the bit: the sum of the weights alone is rounded
    alike = np.full_like(off, (n + 16) * 2.0 ** -24)
    assert (np.abs(got - want) <= ref.tolerance(want, alike, spread, dtype)).all()
    assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("dtype,q_size,k_size,scale", FAR)
@pytest.mark.parametrize("n,scratch", [(300, 0), (2500, 1 << 22)])
def test_large_scores_of_which_one_is_the_largest(dtype, q_size, k_size, scale, n, scratch):
    """All keys point away but one, wherever that stands: the result is its value."""
    rng = np.random.default_rng(6)
    for at in (0, 37, n // 2, n - 1):
        def keys(k):
            k[np.arange(n) != at] ^= 0x8000
            return k
        cache, pages, tables, row = far_case(rng, dtype, k_size, n, keys)
        q = round16(np.broadcast_to((q_size * np.sign(decode64(row, dtype))).astype(np.float32), (1, 2, 128)), dtype)
        hints = (1, n)
        out, lse = attend(cache, tables, [0, 1], [n], bits16(q.reshape(1, -1), dtype), 2, scale, scratch=scratch, hints=hints)
        want, want_lse, off, spread = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), [0, 1], [n], 2, 1, scale)
        got = decode64(host16(out), dtype).reshape(want.shape)
        # the other weights are nothing in any precision (e^-200 and less)
        assert (np.abs(got - want) <= ref.tolerance(want, np.full_like(off, 16 * 2.0 ** -24), spread, dtype)).all(), at
        assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** 80, 2.0 ** 94])
@pytest.mark.parametrize("n,new,scratch", [(200, 1, 0), (600, 4, 0), (150, 40, 0), (4000, 1, 1 << 22)])
def test_values_of_nothing_next_to_the_largest(size, n, new, scratch):
    """Positions whose values are zeros count in the sum of the weights, before and behind values of any size."""
    rng = np.random.default_rng(7)
    for part in (slice(0, n // 2), slice(n // 2, n), slice(0, n - 3), slice(0, n, 2)):
        cache, pages, tables = filled_cache(rng, "bf16", 128, 1, 16, [n])
        v = round16((rng.standard_normal((n, 1, 128)) * size).astype(np.float32), "bf16")
        v[part] = 0
        p = np.arange(n)
        pages.write(1, tables[0, p // 16] * 16 + p % 16, normal(rng, (n, 1, 128), "bf16"), v)
        cache.put(pages)
        q = normal(rng, (new, 2, 128), "bf16")
        hints = (new, n)
        assert not scratch or slices_of(cache, tables, new, 2, hints, scratch) > 1
        out, lse = attend(cache, tables, [0, new], [n], bits16(q.reshape(new, -1), "bf16"), 2, 0.01, scratch=scratch, hints=hints)
        want, want_lse, off, spread = ref.attention(decode64(q, "bf16"), rows_of(pages, tables, 16), [0, new], [n], 2, 1, 0.01)
        got = decode64(host16(out), "bf16").reshape(want.shape)
        # what is held below 2^-31 of the largest value of the tile's rows is lost (here none is, but zeros)
        assert (np.abs(got - want) <= ref.tolerance(want, off, spread, "bf16") + 2.0 ** -31 * np.abs(decode64(v, "bf16")).max()).all()
        assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


def test_a_large_value_of_no_weight_behind_constant_ones():
    """A position that weighs nothing does not take the others' sums with it, however large its value."""
    rng = np.random.default_rng(8)
    n = 300
    for size in (1.0, 2.0 ** 70, 2.0 ** 94):
        for at in (0, 150, n - 1):
            cache, pages, tables = filled_cache(rng, "bf16", 128, 1, 16, [n])
            k = np.broadcast_to(round16(rng.choice((-1.0, 1.0), 128).astype(np.float32), "bf16"), (n, 1, 128)).copy()
            q = round16(np.broadcast_to(decode64(k[0, 0], "bf16").astype(np.float32), (1, 2, 128)), "bf16")
            k[at] ^= 0x8000
            v = np.broadcast_to(round16(np.float32([5.0]), "bf16"), (n, 1, 128)).copy()
            v[at] = round16((rng.standard_normal((1, 128)) * size).astype(np.float32), "bf16")
            p = np.arange(n)
            pages.write(1, tables[0, p // 16] * 16 + p % 16, k, v)
            cache.put(pages)
            # scores of some 192 and -192: the one weighs e^-384, times 2^94 nothing
            out, lse = attend(cache, tables, [0, 1], [n], bits16(q.reshape(1, -1), "bf16"), 2, 1.5)
            assert (decode64(host16(out), "bf16") == 5.0).all(), (size, at)
            _, want_lse, off, _ = ref.attention(decode64(q, "bf16"), rows_of(pages, tables, 16), [0, 1], [n], 2, 1, 1.5)
            assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [1, 7])
def test_logarithms_of_sums_of_equal_weights(dtype, heads):
    """Zero queries over any number of positions whose values are zeros: the logarithm of that number.  Sums of ones are exact, so that the logarithm's own
    rounding (two of its last places, which are of at most 2^-23 next to 1), its product with ln 2 and two additions are all that is off."""
    lens = [*range(1, 40), 100, 555, 1000, 2047, 3000]
    cache = Cache(dtype, 64, 1, 2, 16, 190, fill=0)  # codes, scales and minima of zeros
    tables = np.broadcast_to(np.arange(190), (len(lens), 190)).copy()
    q = np.zeros((len(lens), heads, 64), np.uint16)
    for scratch, hints in ((0, (1, 0)), (1 << 24, (1, 3000)), (0, (40, 0))):
        out, lse = attend(cache, tables, np.arange(len(lens) + 1), lens, bits16(q.reshape(len(lens), -1), dtype), heads, 0.125, scratch=scratch, hints=hints)
        want = np.log(np.array(lens, np.float64))[:, None]
        assert (host(out.float()) == 0).all()
        assert (np.abs(host(lse) - want) <= 2.0 ** -22 + 2.0 ** -22 * want).all(), (scratch, hints, np.abs(host(lse) - want).max())


# ---------------------------------------------------------------------------------------------- slices

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("d,heads,kv_heads,lens,new,window,hints", [
    (128, 4, 2, [6000], [1], 1000, (1, 6000)), (64, 3, 3, [5000], [2], 777, (2, 5000)),
    # ragged: requests of one slice, of some, without rows or positions; more rows and positions than the hint says
    (128, 4, 2, [4100, 2500, 1, 0, 600, 33], [1, 1, 1, 1, 0, 1], 1500, (1, 4100)), (64, 4, 1, [3000, 700], [4, 1], 900, (4, 1200)),
    (64, 2, 2, [3000, 2000], [2, 9], 1300, (2, 3000)),
    # prompts behind long contexts
    (128, 10, 2, [3000, 2200], [40, 40], 1000, (40, 3000)), (64, 4, 4, [2600, 40, 0, 333, 64], [40, 40, 1, 1, 64], 1111, (40, 2600))])
def test_windows_in_slices(dtype, causal, d, heads, kv_heads, lens, new, window, hints):
    """The slices of a row that a window lets see the last positions alone: the first step is not 0, and slices count from it."""
    scratch = 1 << 24
    assert plan_slices(dtype, d, heads, kv_heads, 16, lens, new, hints, scratch, window) > 1
    a = check_attention(dtype, d, heads, kv_heads, 16, lens, new, causal, window, scratch=scratch, hints=hints, seed=31)
    b = check_attention(dtype, d, heads, kv_heads, 16, lens, new, causal, window, scratch=scratch, hints=hints, seed=31)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tiny_scores_and_hidden_pages_in_slices(dtype):
    """All weights alike, those of pages that are not of the cache nothing: whole slices of them, and the ends of others."""
    rng = np.random.default_rng(32)
    n, hints, scratch = 3000, (1, 3000), 1 << 22
    cache, pages, tables = filled_cache(rng, dtype, 128, 1, 16, [n])
    gone = np.r_[3, 40:75, 187]
    tables[0, gone] = -1
    assert slices_of(cache, tables, 1, 2, hints, scratch) > 1
    size, scale = (1e-36, 1e-20) if dtype == "bf16" else (1e-6, 1e-30)
    q = normal(rng, (1, 2, 128), dtype, size)
    out, lse = attend(cache, tables, [0, 1], [n], bits16(q.reshape(1, -1), dtype), 2, scale, scratch=scratch, hints=hints)
    hidden = lambda r: np.isin(np.arange(n) // 16, gone)  # noqa: E731
    want, want_lse, off, spread = ref.attention(decode64(q, dtype), rows_of(pages, tables, 16), [0, 1], [n], 2, 1, scale, hidden=hidden)
    got = decode64(host16(out), dtype).reshape(want.shape)
    assert (np.abs(got - want) <= ref.tolerance(want, off, spread, dtype)).all()
    assert (np.abs(host(lse) - want_lse) <= off + 2.0 ** -22 * (1 + np.abs(want_lse))).all()


def test_calls_in_slices_that_share_a_workspace_in_a_graph():
    """Two captured calls and an eager one use one workspace, one after the other, over replays: each has slices and a join."""
    rng = np.random.default_rng(33)
    lens, hints, nbytes = [3000, 2500], (1, 3000), 1 << 21
    cache, pages, tables = filled_cache(rng, "f16", 128, 2, 16, lens)
    q = bits16(normal(rng, (2, 1024), "f16"), "f16")
    scales = (0.05, 0.3)
    want = [attend(cache, tables, [0, 1, 2], lens, q, 8, s, scratch=nbytes, hints=hints) for s in scales]
    q_starts, kv_lens, t = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"), \
        torch.tensor(tables, device="cuda").int()
    b = sg.make_kv_batch(2, 2, tables.shape[1], q_starts, kv_lens, t, max_q_len=1, max_kv_len=3000)
    plan = sg.sgmv_plan_attention_q4(cache.c, b, 8, 0, 1 << 8, nbytes)
    assert plan.slices > 1 and plan.launches == 2
    work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    outs, sums = [torch.zeros(2, 1024, dtype=torch.float16, device="cuda") for _ in scales], [torch.zeros(2, 8, device="cuda") for _ in scales]

    def call(i, stream):
        sg.sgmv_attention_q4(cache.c, b, 1, outs[i], sums[i], q, 8, 1024, 1024, scales[i], 1, 0, work, nbytes, stream)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(0, stream)
            call(1, stream)
    for i in range(5):
        for x in (*outs, *sums, work):
            x.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        if i % 2:  # the same workspace eagerly behind the replay
            outs[0].record_stream(stream)
            call(0, stream)
        torch.cuda.synchronize()
        for (out, lse), got, got_lse in zip(want, outs, sums):
            assert torch.equal(got, out) and torch.equal(got_lse, lse), i


# ---------------------------------------------------------------------------------------------- scales of the softmax and of rows at the ends of their types

@pytest.mark.parametrize("q_size,scale", [(1e-37, 3.3e38), (1e-38, 3e38), (1e-30, 3.4e38), (1e-39, 1e38)])
def test_softmax_scales_at_the_end_of_fp32(q_size, scale):
    """A scale near fp32's largest, next to rows so small that the scores are ordinary or merely large."""
    check_attention("bf16", 128, 4, 2, 16, [100, 37], [5, 1], q_size=q_size, scale=scale, seed=9)


@pytest.mark.parametrize("q_power,scale_power,fits", [(5, 114, True), (5, 117, False), (60, 59, True), (60, 63, False), (98, -20, True)])
def test_queries_times_the_scale(q_power, scale_power, fits):
    """Rows that times the scale pass 2^120 are NaN where they see positions; others take keys as small as their scores need."""
    rng = np.random.default_rng(10)
    n, d = 60, 128
    cache, pages, tables = filled_cache(rng, "bf16", d, 1, 16, [n])
    k = round16((rng.choice((-1.0, 1.0), (1, 1, d)) * 2.0 ** (10.0 - q_power - scale_power)).astype(np.float32), "bf16")
    p = np.arange(n)
    pages.write(1, tables[0, p // 16] * 16 + p % 16, np.broadcast_to(k, (n, 1, d)), normal(rng, (n, 1, d), "bf16"))
    cache.put(pages)
    # one value at the power itself, the others below it; rows 0 and 1 stand in front of position 0
    q = round16((2.0 ** q_power * np.where(np.arange(d) == 9, 1.0, rng.random((n + 2, 2, d)))).astype(np.float32), "bf16")
    scale = 2.0 ** scale_power
    out, lse = attend(cache, tables, [0, n + 2], [n], bits16(q.reshape(n + 2, -1), "bf16"), 2, scale)
    got, sums = decode64(host16(out), "bf16").reshape(n + 2, 2, d), host(lse)
    assert (got[:2] == 0).all() and np.isneginf(sums[:2]).all()
    if not fits:
        assert np.isnan(got[2:]).all() and np.isnan(sums[2:]).all()
        return
    want, want_lse, off, spread = ref.attention(decode64(q, "bf16"), rows_of(pages, tables, 16), [0, n + 2], [n], 2, 1, scale)
    # keys of the same bytes: scores that are the same to the bit
    assert (np.abs(got - want) <= ref.tolerance(want, np.full_like(off, (n + 16) * 2.0 ** -24), spread, "bf16")).all()
    assert (np.abs(sums[2:] - want_lse[2:]) <= off[2:] + 2.0 ** -17 + 2.0 ** -22 * (1 + np.abs(want_lse[2:]))).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_rows_of_every_size(dtype, d):
    """Rows whose values lie anywhere in their type's range, its smallest numbers among them: bytes of the definition, and back."""
    rng = np.random.default_rng(34)
    n, heads = 400, 2
    low, high = (-133, 126) if dtype == "bf16" else (-25, 15)
    k, v = (round16((rng.standard_normal((n, heads, d)).clip(-1, 1) * 2.0 ** rng.integers(low, high, (n, heads, 1))).astype(np.float32), dtype) for _ in range(2))
    k[::7, 0, 0] ^= 0x8000
    cache = Cache(dtype, d, heads, 2, 16, n // 16)
    slots = rng.permutation(n)
    at = torch.tensor(slots, dtype=torch.int32, device="cuda")
    b = sg.make_kv_batch(1, n, 1, None, None, None, at)
    dk, dv = bits16(k, dtype), bits16(v, dtype)
    sg.sgmv_kv_append_q4(cache.c, b, 1, None, None, dk, dv, heads, heads * d, heads * d, heads * d)
    want = cache.reference()
    want.write(1, slots, k, v)
    # rows of zeros of both signs: the sign of a scale of 0, which meets codes of 0 and a minimum of +0, is that of one of them
    got, held = cache.bytes(), want.bytes.copy()
    for x in (got, held):
        pairs = x[..., 16 * d:].view(np.uint16)
        pairs[..., ::2][pairs[..., ::2] == 0x8000] = 0
    assert np.array_equal(got, held)
    back = [torch.zeros_like(dk), torch.zeros_like(dv)]
    sg.sgmv_kv_read_q4(cache.c, 1, *back, heads * d, at, n)
    for g, w in zip(back, want.rows(1, slots, fp32=True)):
        assert np.array_equal(decode64(host16(g), dtype), decode64(round16(w, dtype), dtype))

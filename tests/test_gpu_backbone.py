"""The 8-bit backbone calls on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import backbone_reference as ref
from helpers import decode64

pytestmark = pytest.mark.gpu
KIND = {"f16": 0, "bf16": 1}
MARK = 0x5A5A  # rows behind the batch and outputs hold this before a call


def _bits(v, dtype):
    return ref.round16(v, dtype)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).to("cuda:0")


def _marked(rows, width, dtype=torch.int16):
    """An output with two rows more than the call has."""
    return torch.full((rows + 2, width), MARK if dtype == torch.int16 else 0x5A, dtype=dtype, device="cuda:0")


def _host(t):
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def _behind(t, n):
    assert torch.all(t[n:] == (MARK if t.dtype == torch.int16 else 0x5A)), "rows behind the batch were written"


def _rows(rng, n, h, dtype, large=0.01):
    v = rng.standard_normal((n, h)) * np.where(rng.random(h) < large, 20.0, 1.0)
    return _bits(v, dtype)


class Q8:
    def __init__(self, n, h):
        self.q = _marked(n, h, torch.int8)
        self.scales = torch.full((n + 2,), -7.0, device="cuda:0")
        self.n = n

    def get(self):
        _behind(self.q, self.n)
        assert torch.all(self.scales[self.n:] == -7.0)
        return _host(self.q)[:self.n], _host(self.scales)[:self.n].astype(np.float64)


WIDTHS = (8, 64, 504, 512, 520, 4096, 5128, 13824, 32768)
ROWS = (1, 2, 67, 600)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("h", WIDTHS)
def test_norm(h, dtype):
    from paper_2310_18547_amd import binding as B
    rng = np.random.default_rng(h)
    for n in ROWS[:3] if h > 8192 else ROWS:
        for has_residual, has_sum, has_out, has_q in ((1, 1, 1, 1), (0, 0, 0, 1), (1, 0, 1, 0), (0, 1, 1, 1)):
            x, r, w = _rows(rng, n, h, dtype), _rows(rng, n, h, dtype), _bits(1 + 0.3 * rng.standard_normal(h), dtype)
            out, total, q8 = _marked(n, h), _marked(n, h), Q8(n, h)
            B.sgmv_rms_norm_q8(KIND[dtype], out if has_out else None, q8.q if has_q else None, q8.scales if has_q else None,
                               total if has_sum else None, _dev(x), _dev(r) if has_residual else None, _dev(w), 1e-5, n, h)
            s, v = ref.norm(x, r if has_residual else None, w, np.float32(1e-5), dtype)
            what = (h, n, has_residual, has_sum, has_out, has_q)
            q, scales = q8.get()
            ref.check_rows(v, _host(out)[:n] if has_out else None, q if has_q else None, scales, dtype, what)
            _behind(out, n if has_out else 0)
            _behind(total, n if has_sum else 0)
            if has_sum:
                # two 16-bit numbers added in fp32: one rounding there (2^-24), one in the store
                off = np.abs(decode64(_host(total)[:n], dtype) - s)
                assert np.all(off <= np.abs(s) * (ref.HALF_STEP[dtype] + 2.0 ** -23) + ref.SMALLEST[dtype]), what


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("h", WIDTHS)
def test_silu_mul_and_quantize(h, dtype):
    from paper_2310_18547_amd import binding as B
    rng = np.random.default_rng(h + 1)
    for n in ROWS[:3] if h > 8192 else ROWS:
        for has_out, has_q in ((1, 1), (0, 1), (1, 0)):
            g, u = _rows(rng, n, h, dtype), _rows(rng, n, h, dtype)
            out, q8 = _marked(n, h), Q8(n, h)
            B.sgmv_silu_mul_q8(KIND[dtype], out if has_out else None, q8.q if has_q else None, q8.scales if has_q else None,
                               _dev(g), _dev(u), n, h)
            q, scales = q8.get()
            _behind(out, n if has_out else 0)
            v = ref.silu_mul(g, u, dtype)
            ref.check_rows(v, _host(out)[:n] if has_out else None, q if has_q else None, scales, dtype, (h, n, has_out, has_q),
                           ref.silu_extra(g, u, v, dtype))
        q8 = Q8(n, h)
        B.sgmv_quantize_q8(KIND[dtype], q8.q, q8.scales, _dev(g), n, h)
        q, scales = q8.get()
        ref.check_rows(decode64(g, dtype), None, q, scales, dtype, (h, n))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_of_zeros_extremes_and_values_that_are_not_finite(dtype):
    from paper_2310_18547_amd import binding as B
    h, n = 264, 10
    rng = np.random.default_rng(5)
    v = rng.standard_normal((n, h))
    big = 65504.0 if dtype == "f16" else 3.3e38
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    v[0] = 0.0
    v[1], v[1, 7] = 0.0, tiny                      # one smallest number
    v[2] = tiny * rng.integers(-9, 10, h)          # subnormal rows
    v[3] = big * np.sign(v[3])                     # squares and their sum leave fp32 (bfloat16)
    v[4] = np.where(rng.random(h) < 0.5, big, 1.0)
    x = _bits(v, dtype)
    inf, nan = (0x7C00, 0x7E00) if dtype == "f16" else (0x7F80, 0x7FC0)
    x[5, 3], x[6, 200], x[7, 0], x[8, 263] = inf, inf | 0x8000, nan, nan | 0x8000
    good, bad = [0, 1, 2, 3, 4, 9], [5, 6, 7, 8]
    w = _bits(np.ones(h) * 0.75, dtype)

    def look(q8, exact, out, what):
        q, scales = q8.get()
        with np.errstate(invalid="ignore"):
            ref.check_rows(exact[good], None if out is None else _host(out)[good], q[good], scales[good], dtype, what)
        assert np.all(np.isnan(scales[bad])) and np.all(q[bad] == 0), what

    q8, out = Q8(n, h), _marked(n, h)
    B.sgmv_rms_norm_q8(KIND[dtype], out, q8.q, q8.scales, None, _dev(x), None, _dev(w), 1e-6, n, h)
    s, exact = ref.norm(x, None, w, np.float32(1e-6), dtype)
    look(q8, exact, out, "norm")
    got = decode64(_host(out)[:n], dtype)
    assert np.all(np.isnan(got[[7, 8]])) and np.isnan(got[5, 3]) and np.isnan(got[6, 200])
    q8 = Q8(n, h)
    B.sgmv_quantize_q8(KIND[dtype], q8.q, q8.scales, _dev(x), n, h)
    look(q8, decode64(x, dtype), None, "quantize")
    ones = np.full((n, h), _bits(np.ones(1), dtype)[0])
    q8, out = Q8(n, h), _marked(n, h)
    B.sgmv_silu_mul_q8(KIND[dtype], out, q8.q, q8.scales, _dev(ones), _dev(x), n, h)
    look(q8, ref.silu_mul(ones, x, dtype), out, "silu")
    # gates at the ends of the range: the activation is the gate itself or zero
    g = np.zeros((2, h))
    g[0], g[1] = big, -big
    q8, out = Q8(2, h), _marked(2, h)
    B.sgmv_silu_mul_q8(KIND[dtype], out, q8.q, q8.scales, _dev(_bits(g, dtype)), _dev(ones[:2]), 2, h)
    got = decode64(_host(out)[:2], dtype)
    assert np.all(got[0] == decode64(_bits(g, dtype), dtype)[0]) and np.all(got[1] == 0.0)
    # eps = 0 is allowed; a row of zeros is then 0 / 0
    q8 = Q8(2, h)
    B.sgmv_rms_norm_q8(KIND[dtype], None, q8.q, q8.scales, None, _dev(x[[0, 9]]), None, _dev(w), 0.0, 2, h)
    q, scales = q8.get()
    assert np.isnan(scales[0]) and np.all(q[0] == 0)
    _, exact = ref.norm(x[[9]], None, w, 0.0, dtype)
    ref.check_rows(exact, None, q[1:], scales[1:], dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_in_place(dtype):
    from paper_2310_18547_amd import binding as B
    n, h = 67, 1032
    rng = np.random.default_rng(11)
    x, r, w = _rows(rng, n, h, dtype), _rows(rng, n, h, dtype), _bits(1 + 0.3 * rng.standard_normal(h), dtype)
    want_out, want_sum, want8 = _marked(n, h), _marked(n, h), Q8(n, h)
    B.sgmv_rms_norm_q8(KIND[dtype], want_out, want8.q, want8.scales, want_sum, _dev(x), _dev(r), _dev(w), 1e-5, n, h)
    for out_is, sum_is in (("x", "r"), ("r", "x"), ("x", None), ("r", None), (None, "x"), (None, "r")):
        t, q8 = {"x": _dev(x), "r": _dev(r), None: None}, Q8(n, h)
        B.sgmv_rms_norm_q8(KIND[dtype], t[out_is], q8.q, q8.scales, t[sum_is], t["x"], t["r"], _dev(w), 1e-5, n, h)
        assert out_is is None or torch.equal(t[out_is], want_out[:n])
        assert sum_is is None or torch.equal(t[sum_is], want_sum[:n])
        assert all(np.array_equal(a, b) for a, b in zip(q8.get(), want8.get()))
    B.sgmv_silu_mul_q8(KIND[dtype], want_out, want8.q, want8.scales, _dev(x), _dev(r), n, h)
    for out_is in ("x", "r"):
        t, q8 = {"x": _dev(x), "r": _dev(r)}, Q8(n, h)
        B.sgmv_silu_mul_q8(KIND[dtype], t[out_is], q8.q, q8.scales, t["x"], t["r"], n, h)
        assert torch.equal(t[out_is], want_out[:n])
        assert all(np.array_equal(a, b) for a, b in zip(q8.get(), want8.get()))


def _dense_inputs(rng, n, h_in, h_outs):
    q = rng.integers(-128, 128, (n, h_in), dtype=np.int8)
    q_scales = (rng.random(n) * 0.02 + 0.001).astype(np.float32)
    ws = [rng.integers(-128, 128, (o, h_in), dtype=np.int8) for o in h_outs]
    w_scales = [(rng.random(o) * 0.02 / np.sqrt(h_in) + 1e-4).astype(np.float32) for o in h_outs]
    return q, q_scales, ws, w_scales


def _dense(dtype, q, q_scales, ws, w_scales, workspace=None, stream=None):
    from paper_2310_18547_amd import binding as B
    n, h_in = q.shape
    ys = [_marked(n, w.shape[0]) for w in ws]
    B.sgmv_dense_q8(KIND[dtype], ys, _dev(q), _dev(q_scales), [_dev(w) for w in ws], [_dev(s) for s in w_scales], n, h_in,
                    [w.shape[0] for w in ws], workspace, 0 if workspace is None else workspace.numel(), stream)
    for y in ys:
        _behind(y, n)
    return [_host(y)[:n] for y in ys]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("h_in", [8, 16, 56, 64, 72, 120, 128, 136, 248, 1000, 4096])
def test_dense_every_tail(h_in, dtype):
    rng = np.random.default_rng(h_in)
    for n in (1, 2, 15, 16, 17, 33, 48, 63, 64, 65, 100, 129, 200, 300):
        for h_outs in ((8,), (264, 16, 72)):
            inputs = _dense_inputs(rng, n, h_in, h_outs)
            for y, w, s in zip(_dense(dtype, *inputs), inputs[2], inputs[3]):
                same = np.array_equal(y, ref.dense(inputs[0], inputs[1], w, s, dtype))
                assert same, (n, h_in, w.shape)


# (tokens, h_in, h_outs, workspace, kernel, LDS, parts of the sum): every kernel of the dense call, an even and an odd number of
# whole steps, with and without a shorter one behind them
EVERY_KERNEL = [
    (1, 1136, (8,), 1, 9, 131072, 1),
    (1, 1152, (8,), 1, 9, 131072, 1),
    (266, 1400, (10552, 5976), 0, 11, 65536, 1),
    (269, 1152, (9600, 7904), 0, 11, 65536, 1),
    (40, 9296, (24, 8408), 1, 11, 65536, 7),
    (36, 10728, (7032, 2848), 1, 11, 65536, 6),
    (67, 1280, (9832, 7320), 0, 10, 163840, 1),
    (67, 1152, (10160, 6576), 1, 10, 163840, 1),
    (2735, 5976, (216,), 1, 10, 163840, 5),
    (75, 5096, (280, 5504), 1, 10, 163840, 4),
    (133, 1280, (9080, 9104), 1, 11, 98304, 1),
    (131, 1160, (4424, 13208), 1, 11, 98304, 1),
    (138, 4424, (8816,), 1, 11, 98304, 3),
    (2704, 10984, (80, 8), 1, 11, 98304, 8),
    (114, 1136, (544,), 0, 9, 98304, 1),
    (81, 1152, (680,), 0, 9, 98304, 1),
    (76, 1144, (1544, 88), 1, 9, 131072, 1),
    (97, 1152, (1160,), 0, 9, 131072, 1),
    (35, 1280, (6184,), 1, 9, 81920, 1),
    (34, 1152, (296, 5816), 1, 9, 81920, 1),
    (516, 1280, (13688, 8), 1, 11, 131072, 1),
    (269, 1160, (9344, 13288), 1, 11, 131072, 1),
    (98, 1280, (16, 2312), 0, 9, 81920, 1),
    (116, 1160, (2000, 48), 1, 9, 81920, 1),
    (1, 1136, (8848,), 1, 9, 81920, 1),
    (1, 1152, (7208, 1024), 1, 9, 81920, 1),
    (33, 1280, (3568, 13200), 0, 9, 163840, 1),
    (68, 1160, (8320, 8), 1, 9, 163840, 1),
    (33, 1280, (28672,), 0, 9, 147456, 1),
    (64, 1160, (25000, 1032), 1, 9, 147456, 1),
    (2865, 1400, (264, 8), 0, 10, 122880, 1),
    (2897, 1152, (8, 280), 0, 10, 122880, 1),
    (2718, 11848, (8,), 1, 10, 122880, 8),
    (2974, 9208, (8,), 1, 10, 122880, 8),
    (131, 1280, (8,), 0, 10, 73728, 1),
    (129, 1152, (8,), 1, 10, 73728, 1),
    (1, 6720, (8,), 1, 10, 73728, 6),
    (6, 6880, (8,), 1, 10, 73728, 6),
    (2862, 1400, (8, 80), 1, 10, 98304, 1),
    (2730, 1152, (72, 8), 1, 10, 98304, 1),
    (2075, 4152, (8,), 1, 10, 98304, 4),
    (2832, 4008, (8,), 1, 10, 98304, 3),
]


@pytest.mark.parametrize("n,h_in,h_outs,scratch,kernel,lds,parts", EVERY_KERNEL)
def test_dense_every_kernel(n, h_in, h_outs, scratch, kernel, lds, parts):
    from paper_2310_18547_amd import binding as B
    workspace = torch.full((16 << 20,), 0x5A, dtype=torch.uint8, device="cuda:0") if scratch else None
    plan = B.sgmv_plan_dense_q8(B.F16, n, h_in, h_outs, workspace, 16 << 20 if scratch else 0)
    assert (plan.kernel, plan.lds_bytes, plan.slices) == (kernel, lds, parts)
    rng = np.random.default_rng(n + h_in)
    for dtype in ("f16", "bf16"):
        inputs = _dense_inputs(rng, n, h_in, h_outs)
        for y, w, s in zip(_dense(dtype, *inputs, workspace=workspace), inputs[2], inputs[3]):
            same = np.array_equal(y, ref.dense(inputs[0], inputs[1], w, s, dtype))
            assert same, (dtype, w.shape)


@pytest.mark.parametrize("n,h_in,h_outs", [(1, 4096, (4096, 4096, 4096)), (7, 13824, (5120,)), (64, 4096, (2752, 2752)),
                                           (65, 11008, (1024,)), (130, 4104, (520, 1032)), (517, 2048, (1024, 256, 256)),
                                           (1031, 1024, (1288,)), (2100, 520, (2048,)), (2100, 512, (2056,)), (64, 131064, (24,)),
                                           (70, 131056, (8,)), (700, 4096, (264,)), (129, 16384, (136,))])
def test_dense_shapes(n, h_in, h_outs):
    rng = np.random.default_rng(n + h_in)
    inputs = _dense_inputs(rng, n, h_in, h_outs)
    want = [ref.dense(inputs[0], inputs[1], w, s, "bf16") for w, s in zip(inputs[2], inputs[3])]
    for scratch in (None, torch.empty(16 << 20, dtype=torch.uint8, device="cuda:0"),
                    torch.empty(100 << 10, dtype=torch.uint8, device="cuda:0")):
        for y, v in zip(_dense("bf16", *inputs, workspace=scratch), want):
            same = np.array_equal(y, v)
            assert same, (n, h_in, h_outs)


def test_dense_extreme_sums_and_scales():
    """The largest sums that int8 gives at the widest input, and scales that are zero, huge, not finite."""
    n, h_in, o = 6, 131064, 16
    q = np.full((n, h_in), -128, np.int8)
    w = np.full((o, h_in), -128, np.int8)
    w[1] = 127
    w[2, ::2] = 127
    q_scales = np.array([1e-9, 0.0, np.nan, np.inf, 1e30, 1e-38], np.float32)
    w_scales = np.full(o, 1e-3, np.float32)
    w_scales[3], w_scales[4], w_scales[5] = 0.0, 1e-30, np.inf
    for dtype in ("f16", "bf16"):
        got, want = _dense(dtype, q, q_scales, [w], [w_scales])[0], ref.dense(q, q_scales, w, w_scales, dtype)
        a, b = decode64(got, dtype), decode64(want, dtype)
        assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])
        assert np.all(np.isnan(a[2]))


def test_dense_one_call_equals_a_call_per_projection_and_repeats():
    rng = np.random.default_rng(3)
    for n in (3, 64, 150, 900):
        q, qs, ws, ss = _dense_inputs(rng, n, 1536, (512, 264, 512, 8, 1024, 40, 16, 136))
        joint = _dense("f16", q, qs, ws, ss)
        again = _dense("f16", q, qs, ws, ss)
        for i in range(8):
            one = _dense("f16", q, qs, [ws[i]], [ss[i]])[0]
            assert np.array_equal(joint[i], one) and np.array_equal(joint[i], again[i])


def test_offsets_past_32_bits():
    from paper_2310_18547_amd import binding as B
    gen = torch.Generator(device="cuda:0").manual_seed(1)

    def ints(*shape):
        return torch.randint(-127, 128, shape, generator=gen, dtype=torch.int8, device="cuda:0")

    def check(y, q, qs, w, ws, rows, cols):
        want = ref.dense(_host(q[rows]), _host(qs[rows]), _host(w[cols]), _host(ws[cols]), "bf16")
        assert np.array_equal(_host(y[rows][:, cols].contiguous()), want)

    for n, h_in, h_out in ((3, 16384, 139264), (70, 16384, 139264), (300000, 64, 8192), (40000, 65536, 64)):
        q, w = ints(n, h_in), ints(h_out, h_in)
        qs = torch.rand(n, generator=gen, device="cuda:0") * 0.01
        ws = torch.rand(h_out, generator=gen, device="cuda:0") * 0.001
        y = torch.empty(n, h_out, dtype=torch.int16, device="cuda:0")
        B.sgmv_dense_q8(B.BF16, [y], q, qs, [w], [ws], n, h_in, [h_out])
        rows, cols = [0, n // 2, n - 1], [0, 7, h_out // 2, h_out - 9, h_out - 1]
        check(y, q, qs, w, ws, rows, cols)
        del q, w, y
    n, h = 70000, 32768
    x = torch.empty(n, h, dtype=torch.bfloat16, device="cuda:0").normal_(generator=gen)
    q, scales = torch.empty(n, h, dtype=torch.int8, device="cuda:0"), torch.empty(n, device="cuda:0")
    B.sgmv_quantize_q8(B.BF16, q, scales, x, n, h)
    rows = [0, n // 2, n - 1]
    v = x[rows].double().cpu().numpy()
    ref.check_rows(v, None, _host(q[rows]), _host(scales[rows]).astype(np.float64), "bf16")


def test_two_streams_at_once():
    """Dense calls on two streams, with workspaces of their own, do not disturb each other."""
    from paper_2310_18547_amd import binding as B
    rng = np.random.default_rng(21)
    n, h_in, h_out = 100, 8192, 1032
    assert B.sgmv_plan_dense_q8(B.F16, n, h_in, [h_out], 0x10000, 16 << 20).slices > 1
    jobs = []
    for _ in range(2):
        q, qs, ws, ss = _dense_inputs(rng, n, h_in, (h_out,))
        jobs.append(dict(want=ref.dense(q, qs, ws[0], ss[0], "f16"), q=_dev(q), qs=_dev(qs), w=_dev(ws[0]), s=_dev(ss[0]),
                         y=[_marked(n, h_out) for _ in range(20)], stream=torch.cuda.Stream(device="cuda:0"),
                         scratch=torch.empty(16 << 20, dtype=torch.uint8, device="cuda:0")))
    torch.cuda.synchronize()
    for i in range(20):
        for j in jobs:
            B.sgmv_dense_q8(B.F16, [j["y"][i]], j["q"], j["qs"], [j["w"]], [j["s"]], n, h_in, [h_out], j["scratch"], 16 << 20, j["stream"])
    torch.cuda.synchronize()
    for j in jobs:
        for y in j["y"]:
            _behind(y, n)
            same = np.array_equal(_host(y)[:n], j["want"])
            assert same


def test_streams_graphs_and_repeated_calls():
    """A layer's calls on a stream of their own, captured, replayed with new inputs in the same buffers."""
    from paper_2310_18547_amd import binding as B
    rng = np.random.default_rng(9)
    n, h, ffn = 70, 520, 1048
    x, r, w = _dev(_rows(rng, n, h, "f16")), _dev(_rows(rng, n, h, "f16")), _dev(_bits(np.ones(h), "f16"))
    wg, wu = (_dev(rng.integers(-128, 128, (ffn, h), dtype=np.int8)) for _ in range(2))
    sg = _dev((rng.random(ffn) * 1e-3).astype(np.float32))
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")

    def buffers():
        return {"out": _marked(n, h), "sum": _marked(n, h), "a": Q8(n, h), "g": _marked(n, ffn), "u": _marked(n, ffn),
                "act": _marked(n, ffn), "b": Q8(n, ffn)}

    def run(t, stream):
        B.sgmv_rms_norm_q8(B.F16, t["out"], t["a"].q, t["a"].scales, t["sum"], x, r, w, 1e-5, n, h, stream)
        B.sgmv_dense_q8(B.F16, [t["g"], t["u"]], t["a"].q, t["a"].scales, [wg, wu], [sg, sg], n, h, [ffn, ffn], scratch,
                        scratch.numel(), stream)
        B.sgmv_silu_mul_q8(B.F16, t["act"], t["b"].q, t["b"].scales, t["g"], t["u"], n, ffn, stream)

    stream = torch.cuda.Stream(device="cuda:0")
    eager, captured = buffers(), buffers()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        run(captured, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run(captured, torch.cuda.current_stream())
    for i in range(4):
        x.copy_(_dev(_rows(rng, n, h, "f16")))
        torch.cuda.synchronize()
        run(eager, None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in eager:
            a, b = (eager[k], captured[k]) if k not in "ab" else (eager[k].q, captured[k].q)
            assert torch.equal(a, b), (i, k)
        assert torch.equal(eager["b"].scales, captured["b"].scales)

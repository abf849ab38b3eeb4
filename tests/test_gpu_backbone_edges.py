"""Edges of the 8-bit backbone calls on the GPU: sums of a few steps in every dense kernel, norms of the smallest rows."""
import numpy as np
import pytest
import torch

import backbone_reference as ref
from test_gpu_backbone import KIND, Q8, _behind, _bits, _dense_inputs, _dev, _host, _marked

pytestmark = pytest.mark.gpu

# (tokens, h_in, h_outs, kernel, LDS): the tile kernels with one whole step of 128 up to as many as their rings have places (the
# large ones, whose schedule spans two steps, up to five), the wide kernels for few tokens with one chunk up to two for every wave;
# each with and without a shorter step behind them
FEW_STEPS = [
    (132, 128, (8,), 10, 73728),
    (134, 136, (8,), 10, 73728),
    (129, 256, (8,), 10, 73728),
    (129, 264, (8,), 10, 73728),
    (137, 384, (8,), 10, 73728),
    (131, 392, (8,), 10, 73728),
    (129, 512, (8,), 10, 73728),
    (132, 520, (8,), 10, 73728),
    (130, 640, (8,), 10, 73728),
    (134, 648, (8,), 10, 73728),
    (129, 768, (8,), 10, 73728),
    (130, 776, (8,), 10, 73728),
    (1603, 128, (200, 40, 8), 10, 98304),
    (1802, 184, (152, 16, 8), 10, 98304),
    (1999, 256, (216, 8), 10, 98304),
    (1955, 376, (8, 152, 8), 10, 98304),
    (1760, 384, (224, 24), 10, 98304),
    (1820, 448, (72, 8, 88), 10, 98304),
    (1493, 512, (224, 24, 24), 10, 98304),
    (1346, 520, (24, 144, 96), 10, 98304),
    (1153, 640, (288, 8, 8), 10, 98304),
    (1785, 696, (32, 8, 152), 10, 98304),
    (1365, 768, (8, 8, 288), 10, 98304),
    (1701, 888, (16, 16, 152), 10, 98304),
    (1621, 128, (16, 600), 10, 122880),
    (1641, 192, (16, 432, 80), 10, 122880),
    (1681, 256, (72, 152, 304), 10, 122880),
    (1725, 328, (72, 400, 8), 10, 122880),
    (1647, 384, (16, 472, 16), 10, 122880),
    (1371, 440, (592, 16, 24), 10, 122880),
    (1947, 512, (8, 104, 328), 10, 122880),
    (1986, 568, (24, 16, 408), 10, 122880),
    (1680, 640, (8, 8, 504), 10, 122880),
    (1809, 712, (72, 336, 56), 10, 122880),
    (1916, 768, (352, 24, 72), 10, 122880),
    (1820, 776, (472, 32), 10, 122880),
    (1226, 128, (200, 904, 440), 10, 163840),
    (1963, 200, (200, 584, 176), 10, 163840),
    (1756, 256, (16, 880, 232), 10, 163840),
    (1947, 312, (224, 8, 720), 10, 163840),
    (1723, 384, (808, 8, 304), 10, 163840),
    (1956, 504, (8, 8, 976), 10, 163840),
    (1644, 512, (1232,), 10, 163840),
    (1606, 520, (1040, 168), 10, 163840),
    (1955, 640, (1064,), 10, 163840),
    (1710, 696, (32, 80, 968), 10, 163840),
    (1853, 768, (200, 96, 768), 10, 163840),
    (1970, 776, (856, 120, 8), 10, 163840),
    (87, 128, (12032, 20808, 192), 11, 65536),
    (288, 136, (16344, 600, 8), 11, 65536),
    (258, 256, (216, 16800), 11, 65536),
    (260, 264, (16480,), 11, 65536),
    (262, 384, (240, 576, 15520), 11, 65536),
    (258, 392, (144, 12992, 3784), 11, 65536),
    (1303, 512, (4944, 160, 144), 11, 65536),
    (1300, 584, (5264, 24), 11, 65536),
    (1347, 640, (4904, 432), 11, 65536),
    (1560, 648, (4304, 56, 168), 11, 65536),
    (129, 128, (13504, 3096), 11, 98304),
    (132, 136, (17544, 256, 40), 11, 98304),
    (1983, 256, (1896, 32, 96), 11, 98304),
    (1091, 312, (3232, 8, 136), 11, 98304),
    (1773, 384, (88, 2168, 80), 11, 98304),
    (1568, 392, (80, 2208, 8), 11, 98304),
    (1427, 512, (440, 472, 1736), 11, 98304),
    (1719, 632, (8, 1560, 520), 11, 98304),
    (1489, 640, (200, 2376, 16), 11, 98304),
    (1580, 648, (8, 2192, 88), 11, 98304),
    (153, 128, (8, 8104, 24968), 11, 131072),
    (259, 136, (20816, 272, 1288), 11, 131072),
    (1033, 256, (7064, 16), 11, 131072),
    (1538, 320, (24, 4712, 192), 11, 131072),
    (1025, 384, (7240,), 11, 131072),
    (1692, 392, (24, 4640), 11, 131072),
    (1941, 512, (3120, 1088), 11, 131072),
    (1937, 568, (8, 4128), 11, 131072),
    (1837, 640, (456, 248, 3720), 11, 131072),
    (1922, 704, (24, 40, 4024), 11, 131072),
    (33, 128, (3664, 11376, 1456), 9, 163840),
    (98, 136, (6368, 16), 9, 163840),
    (34, 256, (24, 16544), 9, 163840),
    (68, 264, (8632,), 9, 163840),
    (43, 384, (1184, 520, 14720), 9, 163840),
    (66, 392, (7464, 1136, 80), 9, 163840),
    (40, 512, (8, 1728, 14728), 9, 163840),
    (76, 520, (8264, 128, 88), 9, 163840),
    (37, 640, (64, 8, 16296), 9, 163840),
    (73, 648, (4272, 128, 3960), 9, 163840),
    (57, 768, (16544, 16), 9, 163840),
    (72, 776, (8528,), 9, 163840),
    (41, 896, (16, 16456), 9, 163840),
    (68, 904, (216, 8032, 184), 9, 163840),
    (37, 1024, (16392,), 9, 163840),
    (69, 1032, (40, 8200), 9, 163840),
    (18, 128, (160, 688, 24512), 9, 147456),
    (71, 136, (8, 12272), 9, 147456),
    (17, 256, (24016, 824), 9, 147456),
    (80, 264, (12328,), 9, 147456),
    (17, 384, (24920,), 9, 147456),
    (72, 392, (6120, 6824), 9, 147456),
    (19, 512, (23496, 1560), 9, 147456),
    (33, 520, (328, 16, 24488), 9, 147456),
    (18, 640, (24768,), 9, 147456),
    (35, 648, (72, 14112, 10760), 9, 147456),
    (17, 768, (24584,), 9, 147456),
    (34, 776, (16, 25520, 8), 9, 147456),
]


@pytest.mark.parametrize("n,h_in,h_outs,kernel,lds", FEW_STEPS)
def test_dense_few_steps(n, h_in, h_outs, kernel, lds):
    from paper_2310_18547_amd import binding as B
    plan = B.sgmv_plan_dense_q8(B.F16, n, h_in, h_outs)
    assert (plan.kernel, plan.lds_bytes, plan.slices) == (kernel, lds, 1)
    q, q_scales, ws, w_scales = _dense_inputs(np.random.default_rng(n + h_in), n, h_in, h_outs)
    device = _dev(q), _dev(q_scales), [_dev(w) for w in ws], [_dev(s) for s in w_scales]
    for dtype in ("f16", "bf16"):
        ys = [_marked(n, o) for o in h_outs]
        B.sgmv_dense_q8(KIND[dtype], ys, *device, n, h_in, h_outs)
        for y, w, s in zip(ys, ws, w_scales):
            _behind(y, n)
            same = np.array_equal(_host(y)[:n], ref.dense(q, q_scales, w, s, dtype))
            assert same, (dtype, w.shape)


@pytest.mark.parametrize("h", [8, 520, 4096, 32768])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 1e-42, 1e-38, 1e-32, 1e-29])
def test_norm_of_rows_whose_squares_leave_fp32(eps, h):
    """bfloat16 rows down to the smallest numbers: their squares have few bits in fp32 or none, the normed rows all of them."""
    from paper_2310_18547_amd import binding as B
    rng = np.random.default_rng(h)
    size = 10.0 ** np.concatenate([-np.arange(15.0, 40.0, 0.5), [3, 18.5, 19.5, 37]])[:, None]
    n = size.size
    v = rng.standard_normal((n, h)) * size
    v[:, 0] = np.maximum(size[:, 0], 2.0 ** -133)  # no row of zeros
    v[5], v[5, h // 2] = 0.0, 2.0 ** -133          # the smallest number alone
    r = v * rng.standard_normal((n, h))
    r[:, 0], r[5] = 0.0, 0.0
    x, r = _bits(v, "bf16"), _bits(r, "bf16")
    w = _bits(1 + 0.3 * rng.standard_normal(h), "bf16")
    for residual in (None, r):
        out, q8 = _marked(n, h), Q8(n, h)
        B.sgmv_rms_norm_q8(B.BF16, out, q8.q, q8.scales, None, _dev(x), None if residual is None else _dev(r), _dev(w), eps, n, h)
        _, exact = ref.norm(x, residual, w, np.float64(np.float32(eps)), "bf16")
        assert np.all(np.isfinite(exact))
        q, scales = q8.get()
        ref.check_rows(exact, _host(out)[:n], q, scales, "bf16", (eps, h))


def test_dense_of_more_tiles_than_a_launch_takes():
    """Several launches over ranges of tokens, every row of every projection against the whole sums."""
    from paper_2310_18547_amd import binding as B
    n, h_in, h_out, projections = (1 << 28) + 300, 8, 8, 8
    assert B.sgmv_plan_dense_q8(B.BF16, n, h_in, [h_out] * projections).launches > 1
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    period = (1 << 20) + 7                          # odd: equal rows lie differently in every tile and launch
    some = torch.randint(-128, 128, (period, h_in), generator=gen, dtype=torch.int8, device="cuda:0")
    some_scales = torch.rand(period, generator=gen, device="cuda:0") + 0.01
    q = torch.empty(n, h_in, dtype=torch.int8, device="cuda:0")
    q_scales = torch.empty(n, device="cuda:0")
    for lo in range(0, n, period):
        rows = min(period, n - lo)
        q[lo:lo + rows], q_scales[lo:lo + rows] = some[:rows], some_scales[:rows]
    ws = [torch.randint(-128, 128, (h_out, h_in), generator=gen, dtype=torch.int8, device="cuda:0") for _ in range(projections)]
    w_scales = [torch.rand(h_out, generator=gen, device="cuda:0") + 0.01 for _ in range(projections)]
    ys = [torch.full((n + 2, h_out), 7.0, dtype=torch.bfloat16, device="cuda:0") for _ in range(projections)]
    B.sgmv_dense_q8(B.BF16, ys, q, q_scales, ws, w_scales, n, h_in, [h_out] * projections)
    for y, w, s in zip(ys, ws, w_scales):
        # whole sums below 2^18 are exact in fp32 in any order; then the scales one after the other and one rounding
        want = (((some.float()[:, None, :] * w.float()[None]).sum(2) * some_scales[:, None]) * s).to(torch.bfloat16)
        for lo in range(0, n, period):
            rows = min(period, n - lo)
            same = torch.equal(y[lo:lo + rows], want[:rows])
            assert same, lo
        assert torch.all(y[n:] == 7.0)

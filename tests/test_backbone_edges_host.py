"""Edges of the 8-bit backbone calls without a GPU."""
import pytest
import torch  # noqa: F401  (before the library: a process has one HIP runtime, torch's)

import paper_2310_18547_amd as sg

FAKE = 0x10000   # a non-null, aligned address that is never dereferenced on these paths
OK, NULL, SHAPE, UNSUPPORTED, ALIGN = 0, 1, 2, 3, 4


@pytest.mark.parametrize("n", [1, 5, 128, 129, 1 << 14, 1 << 20, 1 << 27, 1 << 28, (1 << 28) + 300, (1 << 29) + 8, 1 << 30])
def test_plan_dense_takes_every_batch_within_the_stated_limits(n):
    """Many narrow projections, a wide one beside narrow ones, the widest: the limit is the number of values, not what a launch takes."""
    for h_outs in ([8], [8] * 2, [8] * 8, [16, 8, 8], [72, 8, 264], [1 << 27, 8], [1 << 27] * 8, [1 << 20] * 3):
        for h_in in (8, 4096):
            for nbytes in (0, 16 << 20):
                rc, p = sg.sgmv_plan_dense_q8(sg.F16, n, h_in, h_outs, FAKE if nbytes else None, nbytes, check=False)
                what = (n, h_in, h_outs, nbytes)
                if n * sum(h_outs) > 1 << 38:
                    assert rc == UNSUPPORTED, what
                    continue
                assert rc == OK and p.launches >= 1 and p.workgroups >= 1, what
                # a launch takes fewer than 2^32 threads, a workgroup of these kernels has 192 at least
                assert p.workgroups * 192 <= p.launches * (1 << 32), what


def test_plan_dense_in_several_launches():
    p = sg.sgmv_plan_dense_q8(sg.F16, 1 << 30, 8, [8, 8])
    assert p.launches > 1 and p.slices == 1
    assert sg.sgmv_plan_dense_q8(sg.F16, 1 << 22, 8, [8] * 8).launches == 1


# buffers of 4 rows of 64: 512 bytes in 16 bits, 256 in 8, 16 of scales; 128 of a norm's weights
ROWS = dict(out=0x10000, q=0x20000, q_scales=0x30000, sum=0x40000, x=0x50000, residual=0x60000, weight=0x70000)
BYTES = dict(out=512, q=256, q_scales=16, sum=512, x=512, residual=512, weight=128)


def _norm(**at):
    a = {**ROWS, **at}
    return sg.sgmv_rms_norm_q8(sg.F16, a["out"], a["q"], a["q_scales"], a["sum"], a["x"], a["residual"], a["weight"], 1e-5, 4, 64,
                               check=False)


def _silu(**at):
    a = {**ROWS, **at}
    return sg.sgmv_silu_mul_q8(sg.F16, a["out"], a["q"], a["q_scales"], a["x"], a["residual"], 4, 64, check=False)


def _quantize(**at):
    a = {**ROWS, **at}
    return sg.sgmv_quantize_q8(sg.F16, a["q"], a["q_scales"], a["x"], 4, 64, check=False)


@pytest.mark.parametrize("call,written,read", [(_norm, ("out", "sum", "q", "q_scales"), ("x", "residual", "weight")),
                                               (_silu, ("out", "q", "q_scales"), ("x", "residual")),
                                               (_quantize, ("q", "q_scales"), ("x",))])
def test_row_calls_refuse_buffers_that_overlap(call, written, read):
    for name in written:
        for other in (*written, *read):
            if other == name:
                continue
            in_place = name in ("out", "sum") and other in ("x", "residual")
            for offset in (0, 16, BYTES[other] - 16, 16 - BYTES[name], -16):
                if offset <= -BYTES[name] or offset >= BYTES[other] or (offset == 0 and in_place):
                    continue
                assert call(**{name: ROWS[other] + offset}) == SHAPE, (name, other, offset)


def _dense(ys, q, q_scales, ws, w_scales, workspace=None, nbytes=0, n=4, h_in=64, h_outs=(64, 32)):
    return sg.sgmv_dense_q8(sg.F16, ys, q, q_scales, ws, w_scales, n, h_in, h_outs, workspace, nbytes, check=False)


def test_dense_refuses_buffers_that_overlap():
    at = [FAKE * i for i in range(1, 9)]  # y, y, q, q_scales, w, w, w_scales, w_scales
    size = [512, 256, 256, 16, 4096, 2048, 256, 128]
    for i in (0, 1):
        for j in range(8):
            for offset in (0, 16, size[j] - 16, 16 - size[i], -16):
                if i == j or offset <= -size[i] or offset >= size[j]:
                    continue
                p = list(at)
                p[i] = p[j] + offset
                assert _dense(p[:2], p[2], p[3], p[4:6], p[6:]) == SHAPE, (i, j, offset)


def test_dense_refuses_partial_sums_over_its_buffers():
    n, h_in, h_outs = 100, 8192, (1032,)
    slices = sg.sgmv_plan_dense_q8(sg.F16, n, h_in, h_outs, FAKE, 16 << 20).slices
    assert slices > 1
    scratch, parts = 1 << 32, 4 * 1032 * n * slices
    far = [(8 + i) << 32 for i in range(5)]       # y, q, q_scales, w, w_scales
    for i, size in enumerate((2 * 1032 * n, h_in * n, 4 * n, 1032 * h_in, 4 * 1032)):
        for at in (scratch, scratch + parts - 16, scratch + 16 - size // 16 * 16):
            p = list(far)
            p[i] = at
            assert _dense([p[0]], p[1], p[2], [p[3]], [p[4]], scratch, 16 << 20, n, h_in, h_outs) == SHAPE, (i, at - scratch)


def test_dense_refuses_a_negative_workspace_size():
    """As an unsigned number it would be room for any partial sums."""
    for nbytes in (-1, -(1 << 40)):
        assert sg.sgmv_plan_dense_q8(sg.F16, 100, 8192, [1032], 1 << 32, nbytes, check=False)[0] == SHAPE
        assert _dense([2 << 32], 3 << 32, 4 << 32, [5 << 32], [6 << 32], 1 << 32, nbytes, 100, 8192, [1032]) == SHAPE

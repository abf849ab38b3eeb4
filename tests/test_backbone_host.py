"""The 8-bit backbone calls without a GPU: what they refuse, and the forms of argument that they take."""
import numpy as np
import pytest
import torch  # noqa: F401  (before the library, which the defaults below load: a process has one HIP runtime, torch's)

import paper_2310_18547_amd as sg

FAKE = 0x10000   # a non-null, aligned address that is never dereferenced on these paths
OK, NULL, SHAPE, UNSUPPORTED, ALIGN = 0, 1, 2, 3, 4


def _norm(dtype=sg.F16, out=FAKE, q=2 * FAKE, q_scales=3 * FAKE, sum=4 * FAKE, x=5 * FAKE, residual=6 * FAKE, weight=7 * FAKE,
          eps=1e-5, n=4, h=64):
    return sg.sgmv_rms_norm_q8(dtype, out, q, q_scales, sum, x, residual, weight, eps, n, h, check=False)


def _silu(dtype=sg.F16, out=FAKE, q=2 * FAKE, q_scales=3 * FAKE, gate=4 * FAKE, up=5 * FAKE, n=4, h=64):
    return sg.sgmv_silu_mul_q8(dtype, out, q, q_scales, gate, up, n, h, check=False)


def _quantize(dtype=sg.F16, q=2 * FAKE, q_scales=3 * FAKE, x=4 * FAKE, n=4, h=64):
    return sg.sgmv_quantize_q8(dtype, q, q_scales, x, n, h, check=False)


def _dense(dtype=sg.F16, ys=(FAKE, 2 * FAKE), q=3 * FAKE, q_scales=4 * FAKE, ws=(5 * FAKE, 6 * FAKE),
           w_scales=(7 * FAKE, 8 * FAKE), n=4, h_in=64, h_outs=(64, 32), workspace=None, nbytes=0):
    return sg.sgmv_dense_q8(dtype, ys, q, q_scales, ws, w_scales, n, h_in, h_outs, workspace, nbytes, check=False)


@pytest.mark.parametrize("call", [_norm, _silu, _quantize])
def test_row_calls_refuse_before_touching_a_device(call):
    assert call(dtype=2) == UNSUPPORTED
    assert call(n=-1) == SHAPE and call(h=0) == SHAPE and call(h=-8) == SHAPE
    assert call(h=12) == UNSUPPORTED and call(h=32776) == UNSUPPORTED
    assert call(n=0) == OK
    assert call(q_scales=None) == NULL and call(q=None) == NULL
    assert call(q=FAKE * 2 + 8) == ALIGN and call(q_scales=FAKE * 3 + 2) == ALIGN


def test_norm_refusals():
    for eps in (-1e-5, float("nan"), float("inf")):
        assert _norm(eps=eps) == UNSUPPORTED
    assert _norm(x=None) == NULL and _norm(weight=None) == NULL and _norm(out=None, q=None, q_scales=None) == NULL
    for name in ("out", "sum", "x", "residual", "weight"):
        assert _norm(**{name: 9 * FAKE + 8}) == ALIGN
    assert _norm(out=4 * FAKE) == SHAPE            # out is sum: one of the two would be lost
    assert _norm(out=5 * FAKE, sum=5 * FAKE) == SHAPE
    assert _norm(sum=7 * FAKE) == SHAPE and _norm(out=7 * FAKE) == SHAPE   # over the weights that other rows read


def test_silu_and_quantize_refusals():
    assert _silu(gate=None) == NULL and _silu(up=None) == NULL and _silu(out=None, q=None, q_scales=None) == NULL
    assert _quantize(x=None) == NULL and _quantize(q=None, q_scales=None) == NULL
    for name in ("out", "gate", "up"):
        assert _silu(**{name: 9 * FAKE + 8}) == ALIGN
    assert _quantize(x=9 * FAKE + 8) == ALIGN


def test_dense_refusals():
    assert _dense(dtype=-1) == UNSUPPORTED
    assert _dense(n=-1) == SHAPE and _dense(h_in=0) == SHAPE and _dense(h_outs=(64, 0)) == SHAPE
    assert _dense(h_in=60) == UNSUPPORTED and _dense(h_outs=(64, 36)) == UNSUPPORTED
    assert _dense(h_in=131072) == UNSUPPORTED      # the sum could leave 32 bits
    many = tuple(FAKE * i for i in range(1, 10))
    assert _dense(ys=many, ws=many, w_scales=many, h_outs=(8,) * 9) == SHAPE
    assert _dense(ys=(), ws=(), w_scales=(), h_outs=()) == OK
    assert _dense(n=0) == OK
    assert _dense(q=None) == NULL and _dense(q_scales=None) == NULL
    assert _dense(ys=(FAKE, None)) == NULL and _dense(ws=(None, FAKE)) == NULL and _dense(w_scales=(FAKE, None)) == NULL
    assert _dense(ys=(FAKE, FAKE)) == SHAPE        # two projections into one y
    assert _dense(q=3 * FAKE + 8) == ALIGN and _dense(ys=(FAKE, 2 * FAKE + 8)) == ALIGN
    assert _dense(ws=(5 * FAKE + 8, FAKE)) == ALIGN and _dense(w_scales=(7 * FAKE + 8, FAKE)) == ALIGN
    assert _dense(workspace=FAKE + 16, nbytes=1 << 20) == ALIGN
    assert sg.lib.sgmv_dense_q8(0, 1, None, FAKE, FAKE, None, None, 4, 64, None, None, 0, None) == NULL


def test_calls_take_keywords_and_every_form_of_argument():
    """Numbers as numpy gives them, lists and tuples; what has no C value raises, and a refused call too."""
    with pytest.raises(sg.SgmvError, match="sgmv_rms_norm_q8"):
        sg.sgmv_rms_norm_q8(sg.F16, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1e-5, n_tokens=np.int64(4), h=np.int32(12))
    with pytest.raises(sg.SgmvError, match="sgmv_dense_q8"):
        sg.sgmv_dense_q8(sg.BF16, [FAKE], FAKE, FAKE, [FAKE], [FAKE], 4, 64, h_outs=np.array([12], np.int32))
    with pytest.raises(sg.SgmvError, match="sgmv_silu_mul_q8"):
        sg.sgmv_silu_mul_q8(sg.F16, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 12)
    with pytest.raises(sg.SgmvError, match="sgmv_quantize_q8"):
        sg.sgmv_quantize_q8(sg.F16, FAKE, FAKE, FAKE, 4, 12, stream=0)
    with pytest.raises(TypeError):
        sg.sgmv_quantize_q8(sg.F16, "q", FAKE, FAKE, 4, 64)
    with pytest.raises(TypeError):
        sg.sgmv_quantize_q8(sg.F16, FAKE, FAKE, FAKE, 4)
    with pytest.raises(TypeError):
        sg.sgmv_rms_norm_q8(sg.F16, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, None, 4, 64)
    assert sg.sgmv_dense_q8(sg.F16, (), FAKE, FAKE, [], (), 4, 64, []) == 0
    assert sg.sgmv_dense_q8(sg.F16, [FAKE, FAKE * 2], FAKE, FAKE, [FAKE], [FAKE, FAKE], 4, 64, [8, 8], check=False) == NULL
    assert sg.DENSE_WORKSPACE_BYTES == 16 << 20


def _plan(n, h_in, h_outs, nbytes=0, **kw):
    return sg.sgmv_plan_dense_q8(sg.F16, n, h_in, h_outs, FAKE if nbytes else None, nbytes, **kw)


def test_plan_dense():
    """Which kernel serves a call: few tokens, small and large tiles, the sum divided where a workspace holds the parts."""
    p = _plan(1, 4096, [4096] * 3)
    assert p.kernel == sg.KERNEL_DENSE_FEW and p.launches == 1 and p.slices == 1 and 0 < p.lds_bytes <= 160 * 1024
    assert _plan(64, 4096, [4096]).kernel == sg.KERNEL_DENSE_FEW
    p = _plan(517, 4096, [4096, 1024, 1024])
    assert p.kernel == sg.KERNEL_DENSE_SMALL and p.workgroups == 5 * (32 + 8 + 8)
    p = _plan(4814, 8192, [28672], 16 << 20)
    assert p.kernel == sg.KERNEL_DENSE_LARGE and p.launches == 1 and p.workgroups == 19 * 112
    alone, joined = _plan(256, 13824, [5120]), _plan(256, 13824, [5120], 16 << 20)
    assert alone.launches == 1 and alone.slices == 1 and joined.launches == 2 and joined.slices > 1
    parts = joined.slices * 256 * 5120 * 4
    assert _plan(256, 13824, [5120], parts).slices == joined.slices and _plan(256, 13824, [5120], parts - 1).slices < joined.slices
    p = _plan(0, 64, [64])
    assert p.kernel == 0 and p.launches == 0
    for bad, rc in ((dict(n=1, h_in=12, h_outs=[8]), UNSUPPORTED), (dict(n=-1, h_in=8, h_outs=[8]), SHAPE),
                    (dict(n=1, h_in=8, h_outs=[12]), UNSUPPORTED), (dict(n=1, h_in=8, h_outs=[8] * 9), SHAPE),
                    (dict(n=(1 << 30) + 8, h_in=8, h_outs=[8]), UNSUPPORTED), (dict(n=1, h_in=8, h_outs=[(1 << 27) + 8]), UNSUPPORTED)):
        assert _plan(**bad, check=False)[0] == rc
    assert sg.lib.sgmv_plan_dense_q8(0, 1, 1, 8, None, None, 0, None) == NULL
    with pytest.raises(sg.SgmvError, match="sgmv_plan_dense_q8"):
        _plan(1, 12, [8])


def test_every_dense_kernel_is_reached_and_fits():
    """Over usual sizes every kernel of the table is the choice for some; grids and LDS stay within what a launch takes."""
    seen = {}
    for n in (1, 3, 16, 17, 32, 33, 45, 48, 64, 65, 96, 128, 200, 256, 384, 517, 768, 1024, 2048, 4814, 1 << 22, 1 << 30):
        for h_in in (8, 1024, 4096, 4104, 13824, 131064):
            for h_outs in ([8], [1024], [2048], [4096], [4096] * 3, [11008] * 2, [5120], [28672], [1 << 27]):
                for nbytes in (0, 16 << 20):
                    rc, p = _plan(n, h_in, h_outs, nbytes, check=False)
                    if rc != 0:
                        assert rc == UNSUPPORTED and n * sum(h_outs) > 1 << 38, (n, h_in, h_outs)
                        continue
                    assert p.lds_bytes <= 160 * 1024 and 1 <= p.slices <= 8 and (p.slices == 1 or nbytes)
                    seen.setdefault((p.kernel, p.lds_bytes), (n, h_in, h_outs))
    # few tokens: rings of 80 K to 160 K; small tiles 64 x 32, 64 x 64, 64 x 128, 128 x 128; large 64 K, 96 K and 128 K
    assert {b >> 10 for k, b in seen if k == sg.KERNEL_DENSE_SMALL} == {72, 96, 120, 160}, seen
    assert {b >> 10 for k, b in seen if k == sg.KERNEL_DENSE_LARGE} == {64, 96, 128}, seen
    assert {b >> 10 for k, b in seen if k == sg.KERNEL_DENSE_FEW} == {80, 96, 128, 144, 160}, seen


def test_quantize_weight():
    from paper_2310_18547_amd.layer import quantize_weight
    w = torch.tensor([[1.0, -2.0, 0.5, 0.0], [0.0] * 4, [1e-44, -1e-44, 3e-45, 0.0], [3e38, -1.0, 1.5e38, 0.0]])
    q, s = quantize_weight(w)
    assert q.dtype == torch.int8 and s.shape == (4,) and (s > 0).all()
    assert q[0].tolist() == [64, -127, 32, 0] and not q[1].any() and not q[2].any() and q[3, 0] == 127  # 63.5: ties to even
    for tiny in range(1, 400):  # multiples of fp32's smallest number
        assert quantize_weight(torch.tensor([[tiny * 2.0 ** -149, -tiny * 2.0 ** -149]]))[0].sum() == 0
    for bad in (float("inf"), float("nan")):
        with pytest.raises(ValueError):
            quantize_weight(torch.tensor([[1.0, bad]]))

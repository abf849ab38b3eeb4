"""The operators of the 8-bit backbone in 64 bits, written from their formulas (numpy, no GPU)."""
import numpy as np

from helpers import decode64

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # relative rounding error of one store
SMALLEST = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half the spacing of the subnormal numbers
# fp32 arithmetic in front of the store.  A row's sum of squares goes through at most 32 additions in a thread, 6 in
# its wave and 16 over the waves, all terms positive: 54 + 1 roundings of 2^-24, half of that through the root; the
# root, two divisions, three products and the addition of the residual are ten more.
FP32 = 40 * 2.0 ** -24


def round16(v, dtype):
    """fp32 values as bit patterns of the 16-bit type, to the nearest, ties to even."""
    v = np.asarray(v, np.float32)
    if dtype == "f16":
        with np.errstate(over="ignore"):
            return v.astype(np.float16).view(np.uint16)
    u = v.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(v), np.uint16(0x7FC0), r)


def norm(x, residual, weight, eps, dtype):
    """(s, n) of rms_norm from 16-bit patterns."""
    s = decode64(x, dtype)
    if residual is not None:
        s = s + decode64(residual, dtype)
    power = np.mean(s * s, axis=1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        return s, s / np.sqrt(power + eps) * decode64(weight, dtype)


def silu_mul(gate, up, dtype):
    g = decode64(gate, dtype)
    with np.errstate(over="ignore", invalid="ignore"):
        return g / (1.0 + np.exp(-g)) * decode64(up, dtype)


def silu_extra(gate, up, v, dtype):
    """What fp32's exp adds to FP32: its argument, gate * log2(e), is off by two roundings of 2^-24 |gate|; and below a gate
    of -88 exp(-gate) leaves fp32's range, the result is zero in place of |gate * up| * 2^-127 at most."""
    g = decode64(gate, dtype)
    return 2.0 ** -23 * np.abs(g) * np.abs(v) + np.abs(g * decode64(up, dtype)) * 2.0 ** -127


def dense(q, q_scales, w, w_scales, dtype):
    """Bit patterns of y: the whole sums exactly, the scales one after the other in fp32, one rounding."""
    sums = q.astype(np.float64) @ w.astype(np.float64).T  # whole numbers below 2^53
    with np.errstate(over="ignore", invalid="ignore"):
        return round16(sums.astype(np.float32) * q_scales.astype(np.float32)[:, None] * w_scales.astype(np.float32), dtype)


def check_rows(v, got_out, q, scales, dtype, what="", extra=0.0):
    """The 16-bit and 8-bit outputs of finite rows against the exact values ``v`` (``extra``: more that each may be off)."""
    extra = np.broadcast_to(extra, v.shape)
    if got_out is not None:
        off = np.abs(decode64(got_out, dtype) - v)
        assert np.all(off <= np.abs(v) * (HALF_STEP[dtype] * (1 + FP32) + FP32) + 1.01 * extra + SMALLEST[dtype]), (what, float(off.max()))
    if q is not None:
        top = np.abs(v).max(axis=1)
        assert np.all(np.abs(scales - top / 127.0) <= top / 127.0 * FP32 + extra.max(axis=1) + 2.0 ** -149), what
        live = top > 0
        assert np.all(q[~live] == 0) and np.all(np.abs(q.astype(np.int32)) <= 127), what
        steps = v[live] / top[live][:, None] * 127.0
        slack = 2 * 127.0 * (FP32 + extra[live].max(axis=1) / top[live])
        assert np.all(np.abs(q[live] - steps) <= 0.5 + slack[:, None]), (what, float(np.abs(q[live] - steps).max()))
        assert np.all(np.abs(q[live].astype(np.int32)).max(axis=1) == 127), what

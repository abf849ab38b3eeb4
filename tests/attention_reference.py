"""The paged 4-bit cache and attention over it in plain Python and 64 bits, written from their definitions (no GPU)."""
import numpy as np

from backbone_reference import HALF_STEP, SMALLEST, round16
from helpers import decode64

NAN16 = {"f16": 0x7FFF, "bf16": 0x7FFF}  # the scale of a row that is not finite


def value32(bits, dtype):
    return decode64(bits, dtype).astype(np.float32)


def quantize(bits, dtype):
    """Rows of 16-bit patterns [..., d] -> (codes uint8 [..., d], scale patterns, minimum patterns [...]): fp32, each step rounded."""
    x = value32(bits, dtype)
    finite = np.isfinite(x).all(-1)
    x = np.where(finite[..., None], x, np.float32(0))
    low, high = x.min(-1) + np.float32(0), x.max(-1)  # a zero is +0
    with np.errstate(over="ignore"):
        span = high - low
    finite &= np.isfinite(span)
    span = np.where(finite, span, np.float32(0))
    scale = round16(span / np.float32(15), dtype)
    s = value32(scale, dtype)[..., None]
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        c = np.where(s > 0, np.clip(np.rint((x - low[..., None]) / s), 0, 15), 0)
    c = np.where(finite[..., None], c, 0)
    return c.astype(np.uint8), np.where(finite, scale, NAN16[dtype]).astype(np.uint16), np.where(finite, round16(low, dtype), 0).astype(np.uint16)


def rotate(bits, dtype, table, positions, dim, adjacent):
    """Rows [t, heads, d] of 16-bit patterns rotated: products and sums in fp32, then rounded."""
    x = value32(bits, dtype)
    half = dim // 2
    cos, sin = table[positions][:, None, :half], table[positions][:, None, half:]
    a, b = (x[..., 0:dim:2], x[..., 1:dim:2]) if adjacent else (x[..., :half], x[..., half:dim])
    with np.errstate(invalid="ignore", over="ignore"):
        na, nb = a * cos - b * sin, b * cos + a * sin
    x = x.copy()
    if adjacent:
        x[..., 0:dim:2], x[..., 1:dim:2] = na, nb
    else:
        x[..., :half], x[..., half:dim] = na, nb
    out = bits.copy()
    out[..., :dim] = round16(x[..., :dim], dtype)
    return out


class Pages:
    """The bytes of a cache: [n_pages][layers][kv heads][page / 16] tiles."""

    def __init__(self, n_pages, layers, heads, page, d, dtype, fill=0):
        self.heads, self.page, self.d, self.dtype = heads, page, d, dtype
        self.bytes = np.full((n_pages, layers, heads, page // 16, 16 * d + 128), fill, np.uint8)

    def write(self, layer, slots, k, v):
        """Rows [t, heads, d] of 16-bit patterns into their slots; slots out of range are skipped."""
        d = self.d
        for which, rows in ((0, k), (1, v)):
            codes, scale, low = quantize(rows, self.dtype)
            packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
            for t, slot in enumerate(slots):
                if not 0 <= slot < self.bytes.shape[0] * self.page:
                    continue
                page, pos = divmod(int(slot), self.page)
                tile, p = self.bytes[page, layer, :, pos // 16], pos % 16
                for j in range(d // 2):
                    at = p * d // 2 + j if which == 0 else 8 * d + (p // 4) * 2 * d + (j // 4) * 16 + (p % 4) * 4 + j % 4
                    tile[:, at] = packed[t, :, j]
                at = 16 * d + 64 * which + 4 * p
                tile[:, at:at + 2] = scale[t][:, None].view(np.uint8)
                tile[:, at + 2:at + 4] = low[t][:, None].view(np.uint8)

    def rows(self, layer, slots, fp32=False):
        """(k, v) that slots stand for, float64 [t, heads, d] (``fp32``: code * scale + minimum rounded to fp32 twice)."""
        slots = np.asarray(slots)
        page, pos = slots // self.page, slots % self.page
        tiles = self.bytes[page, layer, :, pos // 16]  # [t, heads, bytes]
        t, d = np.arange(len(slots)), self.d
        p = pos % 16
        j = np.arange(d // 2)
        out = []
        for which in (0, 1):
            at = p[:, None] * (d // 2) + j if which == 0 else 8 * d + (p[:, None] // 4) * 2 * d + (j // 4) * 16 + (p[:, None] % 4) * 4 + j % 4
            packed = np.take_along_axis(tiles, at[:, None, :].repeat(self.heads, 1), 2)
            codes = np.stack((packed & 15, packed >> 4), -1).reshape(len(slots), self.heads, d)
            at = 16 * d + 64 * which + 4 * p[:, None] + np.arange(4)
            params = np.ascontiguousarray(np.take_along_axis(tiles, at[:, None, :].repeat(self.heads, 1), 2)).view(np.uint16)
            pair = decode64(params, self.dtype)
            if fp32:
                pair = pair.astype(np.float32)
                with np.errstate(over="ignore"):
                    out.append(codes.astype(np.float32) * pair[..., :1] + pair[..., 1:])
            else:
                out.append(codes * pair[..., :1] + pair[..., 1:])
        return out


def assign(page, n_pages, width, n_tokens, new, old, tables, stack, count):
    """What a step makes of the requests' lengths: (status, lens, tables, stack, count, q_starts, slots, positions)."""
    new, old, tables, stack = list(map(int, new)), list(map(int, old)), np.array(tables).copy(), np.array(stack).copy()
    was = (tables.copy(), stack.copy(), int(count))
    status, pushed, needed, rows = 0, 0, 0, 0
    for a, b in zip(new, old):
        if b < 0 or b > width * page or a < -1:
            status |= 8
        elif a >= 0 and a + b > width * page:
            status |= 2
        elif a < 0:
            pushed += -(-b // page)
        else:
            needed += -(-(a + b) // page) - -(-b // page)
            rows += a
    if count < 0 or count + pushed > n_pages:
        status |= 8
    elif needed > count + pushed:
        status |= 1
    if rows > n_tokens:
        status |= 4
    none = np.full(n_tokens, -1)
    if status:
        return status, old, was[0], was[1], was[2], [0] * (len(new) + 1), none, none
    for i, (a, b) in enumerate(zip(new, old)):
        for j in range(-(-b // page) if a < 0 else 0):
            stack[count] = tables[i, j]
            count += 1
    lens, starts, slots, positions = [], [0], none.copy(), none.copy()
    for i, (a, b) in enumerate(zip(new, old)):
        if a >= 0:
            for j in range(-(-b // page), -(-(a + b) // page)):
                count -= 1
                tables[i, j] = stack[count]
        for k in range(max(a, 0)):
            at = tables[i, (b + k) // page]
            if 0 <= at < n_pages:
                slots[starts[-1] + k] = at * page + (b + k) % page
            else:
                status |= 16
            positions[starts[-1] + k] = b + k
        lens.append(0 if a < 0 else a + b)
        starts.append(starts[-1] + max(a, 0))
    return status, lens, tables, stack, count, starts, slots, positions


def attention(q, rows_of, starts, lens, heads, kv_heads, scale, causal=True, window=0, hidden=None):
    """(out, lse, off, spread) in 64 bits.  q float64 [t, heads, d]; rows_of(request, positions) -> (k, v) [n, kv heads, d];
    hidden(request): positions that count as absent.  off [t, heads]: what fp32 may be off in a score and in the sum of the
    weights; spread [t, heads]: the weighted mean of the positions' largest |v|."""
    t, d = q.shape[0], q.shape[2]
    group = heads // kv_heads
    out, lse = np.zeros((t, heads, d)), np.full((t, heads), -np.inf)
    off, spread = np.zeros((t, heads)), np.zeros((t, heads))
    for r in range(len(lens)):
        n = starts[r + 1] - starts[r]
        if n == 0 or lens[r] == 0:
            continue
        k, v = rows_of(r, np.arange(lens[r]))
        gone = np.zeros(lens[r], bool) if hidden is None else hidden(r)
        k, v = k.repeat(group, 1), v.repeat(group, 1)
        for j in range(n):
            pos = lens[r] - n + j
            sees = ~gone
            if causal:
                sees = sees & (np.arange(lens[r]) <= pos)
            if window:
                sees = sees & (np.arange(lens[r]) > pos - window)
            if not sees.any():
                continue
            row = starts[r] + j
            kk, vv = k[sees], v[sees]
            with np.errstate(invalid="ignore", over="ignore"):
                x = np.einsum("hd,phd->hp", q[row], kk) * scale
                top = x.max(-1, keepdims=True)
                w = np.exp(x - top)
                total = w.sum(-1, keepdims=True)
                out[row] = np.einsum("hp,phd->hd", w / total, vv)
                lse[row] = (top + np.log(total))[:, 0]
                # a score is s (sum q c) + m (sum q): s c is at most twice the row's largest |k|, m at most that; d products and their
                # additions, each off by 2^-24; then two roundings of the exponent and one of the exponential
                size = np.einsum("hd,ph->hp", np.abs(q[row]), np.abs(kk).max(-1)) * scale
                off[row] = (3 * size.max(-1) * (d + 4) + 4 * np.abs(x).max(-1) + sees.sum() + 16) * 2.0 ** -24
                spread[row] = np.einsum("hp,ph->h", w / total, np.abs(vv).max(-1))
    return out, lse, off, spread


# The weights times v's scales, next to the largest: one part of 11 bits for bfloat16, two for binary16.
WEIGHT_STEP = {"f16": 2.0 ** -21, "bf16": 2.0 ** -12}


def tolerance(out, off, spread, dtype):
    """What a result may be off: the rounding of the store; weights that are off, in numerator and sum; the parts of the weights, which
    meet codes (times scales) of up to twice v's largest value; the weights that binary16 cannot show next to the largest (2^-25 of
    2^12, a code of 15)."""
    more = (2 * off + 2 * WEIGHT_STEP[dtype]) * spread * 2 + spread * 2.0 ** -31
    return np.abs(out) * HALF_STEP[dtype] * 1.001 + SMALLEST[dtype] + more[..., None]

"""ORACLE - test infrastructure only: a paged KV cache and attention over it.

The cache is a dictionary (sequence, position) -> row per layer in effect; here it is kept
as what the pages' bytes are defined to be (`offset`), position by position and dimension by
dimension, and attention is HeteGen Sec. 2.1, Eq. 1 for tokens at any position:

    out = sum_j softmax(scale * q . K_j)_j V_j   over the positions j <= p that have a page,

in float64 on the stored values.
"""
import numpy as np

from . import decode

SAME, I8, E4M3 = 0, 1, 2
QMAX = {I8: np.float32(127), E4M3: np.float32(448)}


def e4m3_values():
    """Value of each e4m3 code (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F is NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = np.nan if (c & 127) == 127 else -v if c & 128 else v
    return out


def _e4m3_codes(x):
    """Nearest e4m3 code, half to the even code; |x| <= 448."""
    mag = e4m3_values()[:127]
    a = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(mag, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mag[lo], mag[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantise(bits, dtype, fmt):
    """Rows [..., D] of 16-bit patterns -> (codes as uint8 patterns, scales float32)."""
    x = decode(bits, dtype).astype(np.float32)
    with np.errstate(all="ignore"):
        c = (np.max(np.abs(x), axis=-1) * (np.float32(1) / QMAX[fmt])).astype(np.float32)
        q = (x / np.where(c == 0, np.float32(1), c)[..., None]).astype(np.float32)
        ok = (np.isfinite(c) & (c > 0))[..., None]
        q = np.where(ok, q, np.float32(0))
        if fmt == I8:
            codes = np.clip(np.rint(q), -127, 127).astype(np.int8).view(np.uint8)
        else:
            codes = _e4m3_codes(np.clip(q, -448, 448))
        codes = np.where(ok, codes, np.uint8(0))
    return codes, c


def values(codes, fmt, dtype=None):
    """What stored elements stand for, without their scale, in float64."""
    if fmt == SAME:
        return decode(codes, dtype).astype(np.float64)
    if fmt == I8:
        return codes.view(np.int8).astype(np.float64)
    return e4m3_values()[codes]


def record_bytes(fmt, page_size, D):
    return 2 * page_size * D * 2 if fmt == SAME else 2 * page_size * D + 2 * page_size * 4


def offset(fmt, page_size, D, which, pos, d):
    """Byte offset in a record of dimension d of position pos of the page (which: 0 keys, 1 values)."""
    pos, d = np.asarray(pos), np.asarray(d)
    es = 2 if fmt == SAME else 1
    if which == 0:
        tile, i = pos // 16, pos % 16
        if fmt == SAME:
            load, g, e = d // 32, d % 32 // 8, d % 8
        else:
            load, g, e = d // 64, d % 32 // 8, d % 64 // 32 * 8 + d % 8
        return tile * 16 * D * es + load * 1024 + (16 * g + i) * 16 + e * es
    tile, r = pos // 32, pos % 32
    g, e = r % 16 // 4, r // 16 * 4 + r % 4
    if fmt == SAME:
        load, i = d // 16, d % 16
    else:
        load, i, e = d // 32, d % 16, d % 32 // 16 * 8 + e
    return page_size * D * es + tile * 32 * D * es + load * 1024 + (16 * g + i) * 16 + e * es


def scale_offset(page_size, D, which, pos):
    return 2 * page_size * D + which * page_size * 4 + np.asarray(pos) * 4


class Cache:
    """Pages as bytes [n_pages, heads, record], written and read element by element."""

    def __init__(self, heads, D, page_size, n_pages, dtype, fmt, fill=None):
        self.heads, self.D, self.page_size, self.dtype, self.fmt = heads, D, page_size, dtype, fmt
        shape = (n_pages, heads, record_bytes(fmt, page_size, D))
        self.bytes = np.zeros(shape, np.uint8) if fill is None else np.array(fill, np.uint8).reshape(shape)

    def page(self, table_row, pos):
        j = pos // self.page_size
        p = int(table_row[j]) if j < len(table_row) else -1
        return p if 0 <= p < self.bytes.shape[0] else -1

    def write(self, table_row, pos, which, rows):
        """rows [heads, D] (16-bit patterns) at position pos."""
        p = self.page(table_row, pos)
        if p < 0 or pos < 0:
            return
        o = offset(self.fmt, self.page_size, self.D, which, pos % self.page_size, np.arange(self.D))
        if self.fmt == SAME:
            raw = np.ascontiguousarray(rows).view(np.uint8).reshape(self.heads, self.D, 2)
            self.bytes[p][:, o], self.bytes[p][:, o + 1] = raw[..., 0], raw[..., 1]
            return
        codes, c = quantise(rows, self.dtype, self.fmt)
        self.bytes[p][:, o] = codes
        at = int(scale_offset(self.page_size, self.D, which, pos % self.page_size))
        self.bytes[p][:, at:at + 4] = np.ascontiguousarray(c).view(np.uint8).reshape(self.heads, 4)

    def read(self, table_row, first, last, which):
        """float64 [last - first, heads, D] and which positions have a page."""
        out = np.zeros((last - first, self.heads, self.D))
        has = np.zeros(last - first, bool)
        es = 2 if self.fmt == SAME else 1
        for j0 in range(first // self.page_size, -(-last // self.page_size)):
            lo, hi = max(first, j0 * self.page_size), min(last, (j0 + 1) * self.page_size)
            p = self.page(table_row, lo)
            if p < 0:
                continue
            pos = np.arange(lo, hi) % self.page_size
            o = offset(self.fmt, self.page_size, self.D, which, pos[:, None], np.arange(self.D)[None])
            raw = self.bytes[p][:, o]  # [heads, n, D]
            if es == 2:
                raw = raw.astype(np.uint16) | self.bytes[p][:, o + 1].astype(np.uint16) << 8
            v = values(np.ascontiguousarray(raw), self.fmt, self.dtype)
            if self.fmt != SAME:
                at = int(scale_offset(self.page_size, self.D, which, 0))
                sc = np.ascontiguousarray(self.bytes[p][:, at:at + 4 * self.page_size]).view(np.float32)[:, pos]
                with np.errstate(all="ignore"):
                    v = v * sc.astype(np.float64)[..., None]
            out[lo - first:hi - first] = v.transpose(1, 0, 2)
            has[lo - first:hi - first] = True
        return out, has


def attend(q, K, V, pos, has, scale):
    """q [n, Hq, D] at positions pos [n]; K, V [L, Hk, D], has [L].

    Returns out [n, Hq, D] and two numbers per (row, head) that error bounds need: the
    largest sum_d |q_d K_jd| over the visible j, and [n, Hq, D] sum_j softmax_j |V_j|."""
    n, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, qk, mean = np.zeros((n, Hq, D)), np.zeros((n, Hq)), np.zeros((n, Hq, D))
    for i in range(n):
        see = has & (np.arange(K.shape[0]) <= pos[i])
        if not see.any():
            continue
        for h in range(Hq):
            k, v = K[see, h // G], V[see, h // G]
            with np.errstate(all="ignore"):
                s = scale * (k @ q[i, h])
                p = np.exp(s - s.max())
                p = p / p.sum()
                out[i, h] = p @ v
                qk[i, h] = np.max(np.abs(k) @ np.abs(q[i, h]))
                mean[i, h] = p @ np.abs(v)
    return out, qk, mean

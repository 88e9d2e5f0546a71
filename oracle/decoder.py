"""The decoder's attention block in 64 bits, from the definitions of include/ogc_decoder.h (numpy; test infrastructure only)."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rope(x, weight, eps, positions, frequencies, rot, interleaved, magnitude=1.0):
    """x [rows, heads, d] -> the same; weight None: no norm."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    y = x.copy()
    if rot == 0:
        return y
    angle = (np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(frequencies, dtype=np.float64))[:, None, :]
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    return y


def quantize(x):
    """x [..., d] -> codes [..., d], exponents [..., d / 32] (both uint8): the smallest scale 2^(e - 127) at which the largest magnitude of 32
    rounds to 6 or less (2^125 at most: what is larger ends at 6), the nearest code, ties to the even one; 255 and codes 0 where 32 channels hold an infinity or NaN."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    e = np.zeros(top.shape, dtype=np.int64)
    while True:  # up to 7 (exclusive) times the scale rounds to 6
        over = (top >= 7.0 * np.exp2(e - 127.0)) & (e < 252)
        if not over.any():
            break
        e = e + over
    m = np.abs(g) / np.exp2(e - 127.0)[..., None]
    far = np.abs(m[..., None] - E2M1)  # exact in 64 bits
    near = far == far.min(-1, keepdims=True)
    low, high = near.argmax(-1), 7 - near[..., ::-1].argmax(-1)
    code = np.where(low % 2 == 0, low, high) + 8 * np.signbit(g)
    code = np.where(finite[..., None], code, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e, 255).astype(np.uint8)


def values(codes, exponents):
    scale = np.where(exponents == 255, np.nan, np.exp2(exponents.astype(np.float64) - 127.0))
    v = np.where(codes > 7, -1.0, 1.0) * E2M1[codes & 7]
    return v * np.repeat(scale, 32, axis=-1)


class Cache:
    """A cache as bytes [pages][kv_heads][page_size / 32][34 d], one half byte at a time."""

    def __init__(self, data, kv_heads, head_dim, page_size):
        self.data, self.heads, self.d, self.page = data, kv_heads, head_dim, page_size
        assert data.dtype == np.uint8 and data.shape[1:] == (kv_heads, page_size // 32, 34 * head_dim)

    def _place(self, table_row, position):
        e = position // self.page
        page = int(table_row[e]) if e < len(table_row) else -1
        return (page, position % self.page // 32, position % 32) if 0 <= page < len(self.data) else None

    def _bytes(self, t, which):
        c = np.arange(self.d)
        if which == 0:
            return t * (self.d // 2) + c // 2, 4 * (c % 2), 32 * self.d
        return 16 * self.d + c // 32 * 512 + t // 8 * 128 + c % 16 * 8 + c // 16 % 2 * 4 + t % 8 // 2, np.full(self.d, 4 * (t % 2)), 33 * self.d

    def write(self, table_row, position, which, x):
        """x [kv_heads, d]; which: 0 keys, 1 values."""
        at = self._place(table_row, position)
        if at is None:
            return
        page, block, t = at
        codes, exps = quantize(x)
        byte, shift, scales = self._bytes(t, which)
        for h in range(self.heads):
            rec = self.data[page, h, block]
            for nib in (0, 4):
                sel = shift == nib
                rec[byte[sel]] = (rec[byte[sel]] & (0xF0 >> nib)) | (codes[h][sel] << nib)
            rec[scales + 32 * np.arange(self.d // 32) + t] = exps[h]

    def read(self, table_row, position, which):
        """[kv_heads, d] in 64 bits, or None where there is no page."""
        at = self._place(table_row, position)
        if at is None:
            return None
        page, block, t = at
        byte, shift, scales = self._bytes(t, which)
        rec = self.data[page, :, block]
        return values((rec[:, byte] >> shift) & 15, rec[:, scales + 32 * np.arange(self.d // 32) + t])


def attend(q, k, v, visible, scale):
    """q [n, hq, d], k and v [m, hk, d], visible [n, m] bool.  Returns o [n, hq, d] and, of the same shape, the weighted mean of |v| (what
    errors of the weights are measured by), and [n, hq] the largest sum of |q||k| * scale of a row.  Keys that are not seen have no part."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    o, mag, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        for i in range(n):
            see = np.flatnonzero(visible[i])
            if not len(see):
                continue
            kk, vv = k[see, h // group], v[see, h // group]
            with np.errstate(invalid="ignore"):
                s = kk @ q[i, h] * scale
                p = np.exp(s - s.max())
                o[i, h], mag[i, h] = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
            reach[i, h] = (np.abs(kk) @ np.abs(q[i, h]) * scale).max()
    return o, mag, reach

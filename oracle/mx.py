"""A decoder's projections in microscaled formats and the choice of a token, in 64 bits, from the definitions of include/ogc_mx.h and
include/ogc_sample.h (numpy; test infrastructure only)."""
from __future__ import annotations

import numpy as np

MX4, MX8 = 0, 1
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(c & 7) / 8 * 2.0 ** -6 if c >> 3 == 0 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])
CODES = {MX4: E2M1, MX8: E4M3}
SIGN = {MX4: 8, MX8: 128}
# the first magnitude, in units of the scale, that does not round to the largest code any more; the largest exponent byte
OVER = {MX4: (7.0, True), MX8: (464.0, False)}
LAST = {MX4: 252, MX8: 246}


def up(n, to):
    return (n + to - 1) // to * to


def quantize(x, fmt):
    """x [rows, c], c a multiple of 32 -> codes [rows, c], exponents [rows, c / 32] (uint8)."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[0], -1, 32)
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    top, e = np.abs(g).max(-1), np.zeros(g.shape[:2], dtype=np.int64)
    limit, inclusive = OVER[fmt]
    while True:
        edge = limit * np.exp2(e - 127.0)
        over = ((top >= edge) if inclusive else (top > edge)) & (e < LAST[fmt])
        if not over.any():
            break
        e = e + over
    m = np.abs(g) / np.exp2(e - 127.0)[..., None]
    values = CODES[fmt]
    low = np.clip(np.searchsorted(values, m, side="right") - 1, 0, len(values) - 2)
    below, above = m - values[low], values[low + 1] - m  # (exact in 64 bits; beyond the largest code: negative, so the upper one)
    code = np.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low) + SIGN[fmt] * np.signbit(g)
    code = np.where(finite[..., None], code, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e, 255).astype(np.uint8)


def values(codes, exponents, fmt):
    v = CODES[fmt][np.minimum(codes & (SIGN[fmt] - 1), len(CODES[fmt]) - 1)] * np.where(codes & SIGN[fmt], -1.0, 1.0)
    scale = np.where(exponents == 255, np.nan, np.exp2(exponents.astype(np.float64) - 127.0))
    return v * np.repeat(scale, 32, axis=-1)


def places(rows, channels, fmt):
    """Of every (row, channel), rows and channels rounded up: byte and shift of its code, byte of its group's scale."""
    c, r = np.arange(up(channels, 256))[None, :], np.arange(up(rows, 32))[:, None]
    per = 32 if fmt == MX4 else 16  # channels in 16 bytes
    piece = c // per
    byte = (r // 32 * (up(channels, 256) // per) + piece) * 512 + r % 32 * 16 + (c % per // 2 if fmt == MX4 else c % per)
    group = c // 32
    scale = (r // 32 * (up(channels, 256) // 256) + group // 8) * 256 + group % 2 * 128 + r % 32 * 4 + group % 8 // 2
    return byte, (c % 2 * 4 if fmt == MX4 else 0 * c) + 0 * r, scale


def matrix(x, fmt):
    """The bytes (codes, scales) of a matrix with the rows x; rounded-up rows are zero."""
    rows, channels = x.shape
    pad = np.zeros((up(rows, 32), up(channels, 256)))
    pad[:rows, :channels] = x
    codes, e = quantize(pad, fmt)
    byte, shift, scale = places(rows, channels, fmt)
    out = np.zeros(pad.size // (2 if fmt == MX4 else 1), dtype=np.uint8)
    np.bitwise_or.at(out, byte.ravel(), (codes << shift).astype(np.uint8).ravel())
    s = np.zeros(pad.size // 32, dtype=np.uint8)
    s[scale] = np.repeat(e, 32, axis=1)
    return out, s


def codes_of(codes, scales, rows, channels, fmt):
    """(codes, exponents of every channel's group) [rows, padded channels] of a matrix's bytes."""
    byte, shift, scale = places(rows, channels, fmt)
    return ((codes[byte] >> shift) & (2 * SIGN[fmt] - 1))[:rows], scales[scale][:rows]


def read(codes, scales, rows, channels, fmt):
    c, e = codes_of(codes, scales, rows, channels, fmt)
    return values(c, e[:, ::32], fmt)[:, :channels]


def norm(s, weight, eps):
    s = np.asarray(s, dtype=np.float64)
    return s / np.sqrt((s ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)


def gated(a, b):
    with np.errstate(over="ignore", invalid="ignore"):
        return a * b / (1.0 + np.exp(-a))


def sample(row, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """(token, log-probability, margin): margin is how far, relative to the sum it is compared with, the nearest decision was from another one."""
    x = np.asarray(row, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    if not (x > -np.inf).any():
        return -1, -np.inf, np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 0.0, np.inf
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        logs = np.where(x[order] == top, 0.0, (x[order] - top) / temperature)
    exact = np.exp(logs)
    w = np.rint(exact * 2.0 ** 42).astype(np.int64)  # whole numbers: their sums have no rounding
    some = w > 0
    order, w, logs, exact = order[some], w[some], logs[some], exact[some]
    margin = np.inf
    if top_k > 0:
        order, w, logs, exact = order[:top_k], w[:top_k], logs[:top_k], exact[:top_k]
    if top_p < 1:
        sums = np.cumsum(w)
        goal = max(float(top_p), 0.0) * float(sums[-1])
        n = min(int((sums < goal).sum()) + 1, len(w))
        margin = min(margin, np.abs(sums[:-1] - goal).min() / sums[-1] if len(w) > 1 and top_p > 0 else np.inf)
        order, w, logs, exact = order[:n], w[:n], logs[:n], exact[:n]
    if min_p > 0:
        keep = exact >= min(float(min_p), 1.0)
        if min_p < 1:
            margin = min(margin, np.abs(exact - min_p).min())
        order, w, logs = order[keep], w[keep], logs[keep]
    by_index = np.argsort(order)
    order, w, logs = order[by_index], w[by_index], logs[by_index]
    run = np.cumsum(w)
    u = float(uniform) if uniform > 0 else 0.0
    at = min(int((run <= u * float(run[-1])).sum()), len(w) - 1)
    if 0 < u < 1:
        margin = min(margin, np.abs(run[:-1] - u * run[-1]).min() / run[-1] if len(run) > 1 else np.inf)
    return int(order[at]), float(logs[at] - np.log(run[-1] * 2.0 ** -42)), margin

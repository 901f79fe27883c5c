"""References of the serving operators in 64 bits, and how far a correct implementation may be from them."""
import math

import numpy as np

from tests.ops_common import act, attention


def e4m3_values():
    """What the 256 codes stand for, NaN at 127 and 255."""
    c = np.arange(256)
    e, m = c >> 3 & 15, (c & 7).astype(np.float64)
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v[c & 127 == 127] = np.nan
    return np.where(c & 128, -v, v)


def e4m3_rows(x):
    """[..][dim] in 64 bits -> (codes, exponent bytes, values): by search over the codes, ties to the even code."""
    finite = np.where(np.isfinite(x), np.abs(x), 0)
    top = finite.max(axis=-1)
    e = np.full(top.shape, -126)
    for power in range(-126, 121):
        e = np.where(top > 448.0 * 2.0 ** power, power + 1, e)
    s = 2.0 ** e[..., None].astype(np.float64)
    table = e4m3_values()[:127]
    y = np.abs(np.where(np.isfinite(x), x, 0) / s)
    at = np.clip(np.searchsorted(table, y), 1, 126)
    lo, hi = table[at - 1], table[at]
    up = (y - lo > hi - y) | ((y - lo == hi - y) & (at % 2 == 0))
    code = np.where(up, at, at - 1)
    code = np.where(np.isfinite(x), code, 127) | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8), (e + 127).astype(np.uint8), e4m3_values()[code] * s


class Pool:
    """A cache's places as numpy values, [pages][page_size][heads][dim] in 64 bits."""

    def __init__(self, k, v, table, page_size):
        self.k, self.v, self.table, self.size = k, v, np.asarray(table), page_size

    def sequence(self, b, n):
        """(keys, values, which of them are in a page) of the first n tokens of sequence b."""
        pos = np.arange(n)
        col = pos // self.size
        page = np.where(col < self.table.shape[1], self.table[b][np.minimum(col, self.table.shape[1] - 1)], -1)
        there = (page >= 0) & (page < self.k.shape[0])
        page, at = np.where(there, page, 0), pos % self.size
        k, v = self.k[page, at], self.v[page, at]
        return np.where(there[:, None, None], k, 0), np.where(there[:, None, None], v, 0), there


def seen(qn, kn, window, sinks):
    """[qn][kn]: which tokens the query of each new one sees."""
    p, j = np.arange(qn)[:, None] + (kn - qn), np.arange(kn)[None]
    return (j <= p) & ((j < sinks) | (window < 0) | (j >= p - window))


def cache_attention(q, k, v, m, scale):
    """One head of one sequence -> (out, tolerance): as attention over contiguous keys, whose roundings are the same (the scale of
    8-bit values is a power of two: exact). What a query does not see is taken out first, so that it may be NaN."""
    use = m.any(axis=0)
    return attention(q, np.where(use[:, None], k, 0), np.where(use[:, None], v, 0), m, scale)


def lora(x, a, b, adapter, base, ranks, scales, name, f32):
    """-> (y, tolerance), elementwise. An inner sum of K products: every addition (K of them, and a few where parts join) is off by at most 2^-23
    (the matrix cores may truncate) of a partial sum, whose rms is at most that of the whole's terms, sqrt(sum (x a)^2); K of
    them add up as a walk of sqrt(K) steps, and factor 4 takes the largest of up to 10^6. Its two bf16 parts leave 2^-16 of it, the scale 2^-24.
    The outer sum's 2 R products and the base add at most (2 R + 2) 2^-23 of sum |t b| + |base|. Activations have a slope of at most 1.13,
    GELU's formula adds 1.5e-7 of its argument; one rounding of the result (bf16 2^-8 of it, fp32 2^-24)."""
    y = base.copy()
    tol = (2 * a.shape[1] + 2) * 2.0 ** -23 * np.abs(base)
    K = x.shape[1]
    for i in range(a.shape[0]):
        rows = adapter == i
        r = ranks[i]
        if not rows.any() or r == 0:
            continue
        down, up = a[i, :r], b[i, :, :r]
        t = x[rows] @ down.T * scales[i]
        walk = np.sqrt((x[rows] ** 2) @ (down ** 2).T) * abs(scales[i])
        dt = 4 * 2.0 ** -23 * math.sqrt(K + 16) * walk + (2.0 ** -16 + 2.0 ** -23) * np.abs(t)
        y[rows] += t @ up.T
        tol[rows] += dt @ np.abs(up).T + (2 * r + 2) * 2.0 ** -23 * (np.abs(t) @ np.abs(up).T)
    z = act(y, name)
    return z, 1.13 * tol * (1 + 2.0 ** -8) + np.abs(z) * (2.0 ** -24 if f32 else 2.0 ** -8) + (3e-7 * np.abs(y) if name == "gelu" else 0) + 1e-30

"""Float64 definitions of the 8-bit paged cache and its operators, and of token scores (NumPy).

Independent of the GPU package: the cache is held as values (not codes) with its scales, one page
and head at a time, and attention runs one row at a time.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
PAST_RANGE = 1.9375 * 2.0 ** 127        # magnitudes from here on would round to 2^128: as infinities, not a number


def e4m3(x):
    """Nearest e4m3 value, ties to even, of |x| <= 448; NaN stays."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    e = np.where(np.exp2(e) > a, e - 1, e)                 # log2 rounded up at a power of two
    step = np.exp2(np.maximum(e, -6) - 3)
    return np.round(x / step) * step


def page_scale(amax: float) -> float:
    """Least 2^e, e >= -100, with amax <= 448 * 2^e."""
    if amax == 0:
        return 2.0 ** -100
    m, e = math.frexp(amax)                                # amax = m 2^e, 448 = 0.875 * 2^9
    return 2.0 ** max(-100, e - 9 if m <= 0.875 else e - 8)


def head_norm(x, gain, eps):
    return x if gain is None else x * gain / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def turn(x, pos, freq, interleaved=False, magnitude=1.0):
    """Heads x [..., hd] at position `pos` with the leading 2 len(freq) dims turned."""
    n = len(freq)
    lo = 2 * np.arange(n) if interleaved else np.arange(n)
    hi = lo + 1 if interleaved else lo + n
    c, s = np.cos(pos * freq) * magnitude, np.sin(pos * freq) * magnitude
    y = np.array(x, np.float64)
    y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    return y


class Cache:
    """What one layer's cache holds: values [pages][nkv][16][hd] of keys and of values, and scales."""

    def __init__(self, n_pages, nkv, hd):
        self.val = [np.zeros((n_pages, nkv, PAGE, hd)) for _ in range(2)]
        self.scale = [np.zeros((n_pages, nkv)) for _ in range(2)]

    def append(self, table, seq, offset, k, v):
        """k, v [len][nkv][hd] at positions offset .. of sequence `seq`."""
        n = len(k)
        for b in range(offset // PAGE, (offset + n - 1) // PAGE + 1):
            p0 = max(offset, b * PAGE)
            p1 = min(offset + n, (b + 1) * PAGE)
            page, first, last = int(table[seq][b]), p0 - b * PAGE, p1 - b * PAGE
            for which, x in ((0, k), (1, v)):
                for h in range(x.shape[1]):
                    new = x[p0 - offset:p1 - offset, h]
                    new = np.where(np.abs(new) < PAST_RANGE, new, np.nan)
                    fine = new[np.isfinite(new)]
                    s = page_scale(np.abs(fine).max() if fine.size else 0.0)
                    if first > 0 and self.scale[which][page, h] > s:
                        s = self.scale[which][page, h]
                    tile = self.val[which][page, h]
                    tile[:first] = e4m3(tile[:first] / s) * s
                    tile[first:last] = e4m3(new / s) * s
                    self.scale[which][page, h] = s

    def rows(self, table, seq, a, b):
        """Keys and values [b - a][nkv][hd] at positions a .. b - 1."""
        pos = np.arange(a, b)
        page = np.asarray(table)[seq][pos // PAGE]
        return self.val[0][page, :, pos % PAGE], self.val[1][page, :, pos % PAGE]

    def attend(self, table, seq, pos, q, scale, skip=()):
        """Row q [nq][hd] at position `pos`: (output, sum of weights times |value|, largest sum of |q k| scale).
        `skip`: pages whose keys do not count."""
        k, v = self.rows(table, seq, 0, pos + 1)
        keep = np.array([int(np.asarray(table)[seq][p // PAGE]) not in skip for p in range(pos + 1)], bool)
        k, v = k[keep], v[keep]
        nq, nkv = len(q), self.val[0].shape[1]
        out, mag, size = np.zeros(q.shape), np.zeros(q.shape), 0.0
        for h in range(nq):
            g = h // (nq // nkv)
            if len(k) == 0:
                continue
            s = k[:, g] @ q[h] * scale
            size = max(size, float(np.max(np.abs(k[:, g]) @ np.abs(q[h]))) * scale)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[h], mag[h] = p @ v[:, g], p @ np.abs(v[:, g])
        return out, mag, size


def scores(x, tok, n):
    """(logprob, entropy, rank, top ids, top logprobs) of one row of finite or -inf logits."""
    x = np.asarray(x, np.float64)
    m = x.max()
    with np.errstate(invalid="ignore", divide="ignore"):
        lp = x - m - math.log(np.exp(x - m).sum())
        p = np.exp(lp)
        ent = -np.sum(np.where(p > 0, p * lp, 0.0))
    order = np.lexsort((np.arange(len(x)), -x))
    return lp[tok], ent, int(np.nonzero(order == tok)[0][0]), order[:n], lp[order[:n]]

"""Plain restatement of the 8-bit KV cache, in numpy float64 by definition: tables, append, attention, read-back.

A value of the cache is code * scale, with one scale per (page, kv head, K or V): the smallest power of two, not below
2^-126, for which no finite magnitude the page has held exceeds 448 scales.  Codes are e4m3: four significant bits,
spacing at least 2^-9, magnitude at most 448, ties to even; NaN stays NaN, an infinity is stored as 448.
"""
from __future__ import annotations

import numpy as np

P = 16
TOP = 448.0


def e4m3_round(x):
    """Nearest e4m3 value of every element (float64 in and out)."""
    x = np.asarray(x, dtype=np.float64)
    out = np.where(np.isinf(x), np.sign(x) * TOP, x)
    _, e = np.frexp(np.where(np.isfinite(out), out, 0.0))
    step = np.ldexp(1.0, np.maximum(e, -5) - 4)
    out = np.where(np.isnan(out), out, np.rint(out / step) * step)
    return np.where(np.abs(out) > TOP, np.sign(out) * TOP, out)


def e4m3_bits(v):
    """Bit patterns of values that are e4m3 already; NaN gives 0x7F."""
    v = np.asarray(v, dtype=np.float64)
    a = np.abs(np.where(np.isnan(v), 0.0, v))
    _, e = np.frexp(a)
    e = np.where(a == 0, -5, np.maximum(e, -5))       # value = m 2^(e-4), m < 16
    m = np.rint(np.ldexp(a, 4 - e)).astype(np.int64)
    bits = np.where(m < 8, m, ((e + 6) << 3) | (m - 8))
    bits = np.where(np.isnan(v), 0x7F, bits | (np.signbit(v).astype(np.int64) << 7))
    return bits.astype(np.uint8)


def page_scale(x):
    """Smallest power of two s >= 2^-126 with max |finite x| <= 448 s, over the last two axes."""
    a = np.abs(x)
    amax = np.where(np.isfinite(a), a, 0.0).max(axis=(-2, -1))
    s = np.full(amax.shape, 2.0 ** -126)
    while (amax > TOP * s).any():
        s = np.where(amax > TOP * s, 2 * s, s)
    return s


def tables(lens, max_new, free):
    """(cu_seqlens, page_indptr, page list, slot map) of request lengths."""
    cu, indptr, slots = [0], [0], []
    for n in lens:
        first = indptr[-1]
        indptr.append(first + -(-(int(n) + max_new) // P))
        cu.append(cu[-1] + int(n))
        slots += [int(free[first + i // P]) * P + i % P for i in range(int(n))]
    return tuple(np.asarray(a, dtype=np.int32) for a in (cu, indptr, free[:indptr[-1]], slots))


class CacheQ8:
    """Codes (float64 values) and scales of a pool, with the tables of its blocks."""

    def __init__(self, num_pages, heads, d, lens, max_new, free):
        self.codes = np.full((num_pages, heads, 2, P, d), np.nan)
        self.scales = np.full((num_pages, heads, 2), np.nan)
        self.indptr, self.pages = tables(lens, max_new, free)[1:3]
        self.lens = np.zeros(len(lens), dtype=np.int64)

    def page_of(self, b, pos):
        return int(self.pages[self.indptr[b] + pos // P])

    def append(self, b, k, v):
        """Rows [n, heads, d] of block b behind its tokens."""
        x = np.stack([k, v], 2).astype(np.float64)                       # [n, heads, 2, d]
        at, row, n = int(self.lens[b]), 0, len(x)
        while row < n:
            slot = at % P
            take = min(n - row, P - slot)
            pg = self.page_of(b, at)
            new = x[row:row + take].transpose(1, 2, 0, 3)                # [heads, 2, take, d]
            s = page_scale(new)
            if slot:
                s = np.maximum(s, self.scales[pg])
                self.codes[pg, :, :, :slot] = e4m3_round(self.codes[pg, :, :, :slot] * (self.scales[pg] / s)[..., None, None])
            self.codes[pg, :, :, slot:slot + take] = e4m3_round(new / s[..., None, None])
            self.scales[pg] = s
            row, at = row + take, at + take
        self.lens[b] = at

    def rows(self, b, lo, hi):
        """K and V [2, heads, hi - lo, d] of positions lo..hi."""
        out = [self.codes[self.page_of(b, i), :, :, i % P] * self.scales[self.page_of(b, i)][..., None] for i in range(lo, hi)]
        d = self.codes.shape[-1]
        return np.stack(out, 2).transpose(1, 0, 2, 3) if out else np.zeros((2, self.codes.shape[1], 0, d))

    def decode(self, b, q, scale, n=None):
        """(O, spread, shaken) for q [q heads, d] over the first n tokens: O = softmax(scale q k^T) v; spread is the
        same sum over |v|, and shaken the largest sum of |q_i k_i| scale over the keys: what error bounds rest on."""
        n = int(self.lens[b]) if n is None else n
        heads, d = self.codes.shape[1], self.codes.shape[-1]
        qh = np.asarray(q, dtype=np.float64).reshape(heads, -1, d)
        if n == 0:
            z = np.zeros((qh.shape[0] * qh.shape[1], d))
            return z, z, np.zeros((len(z), 1))
        k, v = self.rows(b, 0, n)
        s = scale * (qh @ k.transpose(0, 2, 1))
        w = np.exp(s - s.max(2, keepdims=True))
        w /= w.sum(2, keepdims=True)
        shaken = scale * (np.abs(qh) @ np.abs(k).transpose(0, 2, 1)).max(2)
        return (w @ v).reshape(-1, d), (w @ np.abs(v)).reshape(-1, d), shaken.reshape(-1, 1)

    def floors(self, b, q, scale):
        """(score_floor, weight_floor) for q over the block's tokens: what a kernel may be off on top of decode_tolerance's
        relative terms if it holds queries and weights in f16.

        Queries: scaled by a power of two so that the row's largest magnitude is at least 2^7; an element then is off by
        half of f16's smallest step, 2^-25, at most, which is 2^-32 of the row's largest, times |k| in the score.
        Weights: with V's scale and with 2^6 at the largest p_j * scale_j that the sum has met, off by 2^-25 at most where
        they are subnormal: 2^-31 max_j(p_j scale_j) in all, times |code| in the sum."""
        n, (heads, d) = int(self.lens[b]), (self.codes.shape[1], self.codes.shape[-1])
        qh = np.asarray(q, dtype=np.float64).reshape(heads, -1, d)
        k, _ = self.rows(b, 0, n)
        pages = [self.page_of(b, i) for i in range(n)]
        codes = np.stack([self.codes[p, :, 1, i % P] for i, p in enumerate(pages)], 1)       # [heads, n, d]
        vs = np.stack([self.scales[p, :, 1] for p in pages], 1)                              # [heads, n]
        s = scale * (qh @ k.transpose(0, 2, 1))
        w = np.exp(s - s.max(2, keepdims=True))
        w /= w.sum(2, keepdims=True)
        top = (w * vs[:, None]).max(2)                                                       # [heads, group]
        weight = 2.0 ** -31 * top[..., None] * np.abs(codes).sum(1)[:, None]
        score = 2.0 ** -32 * scale * np.abs(qh).max(2) * np.abs(k).sum(2).max(1)[:, None]
        return score.reshape(-1, 1), weight.reshape(-1, d)


def decode_tolerance(o, spread, shaken, d, score_floor=0.0, weight_floor=0.0):
    """How far a decode kernel with bf16 output, 32-bit sums and 11-bit weights may be off, element by element.

    bf16 output: half a step, 2^-8 |o|.  Weights rounded to f16: 2^-11 of each term.  A score is a sum of d products in
    32 bits, off by at most d 2^-24 of the sum of magnitudes, and its scaling and shift before the exponential add a few
    2^-24 of the score: its error e enters numerator and denominator, 2 e of each term.  The exponential itself and the
    32-bit sums and joins of the partials: 2^-18 of each term.  The floors are those of CacheQ8.floors, for inputs whose
    large values do not meet the dimension looked at."""
    e = (d + 8) * 2.0 ** -24 * shaken + score_floor
    return 2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2 * e + 2.0 ** -18) * spread + weight_floor + 2.0 ** -133

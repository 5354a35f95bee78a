"""Plain restatement of rotary positions and latent attention, in numpy float64 by definition.

Rotary positions: pair i of a rotated part of R elements is turned by position * f_i.  The latent cache holds one row
[c | r] per token: c the normalised latent vector, r the positional key turned to the token's position.  The absorbed form
scores a row with scale (q_c . c + q_r . r) and sums the c; the expanded form has keys [k_nope | r] and values per head.
"""
from __future__ import annotations

import math

import numpy as np

P = 16


# ---------------------------------------------------------------- rotary positions

def frequencies(R, base, scaling="none", factor=1.0, fast=32.0, slow=1.0, trained=4096):
    """f_i of the R/2 pairs, radians per position."""
    i = np.arange(R // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (R / (R - 2))
    f = base ** (-2.0 * i / R)
    if scaling == "all":
        return f / factor
    if scaling == "parts":
        at = lambda t: R * math.log(trained / (2 * math.pi * t)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), R - 1)
        keep = 1 - np.clip((i - lo) / max(hi - lo, 0.001), 0, 1)
    elif scaling == "waves":
        keep = np.clip((trained * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
    else:
        return f
    return f * keep + f / factor * (1 - keep)


def turn(x, positions, f, interleaved, amplitude=1.0, inverse=False):
    """x [..., R] turned to `positions` (whatever broadcasts over the leading axes)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.asarray(positions, dtype=np.float64)[..., None] * f
    c, s = np.cos(a) * amplitude, np.sin(a) * (-amplitude if inverse else amplitude)
    half = x.shape[-1] // 2
    u, v = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    y = np.empty(np.broadcast_shapes(x.shape, a.shape[:-1] + (2 * half,)))
    if interleaved:
        y[..., 0::2], y[..., 1::2] = u * c - v * s, v * c + u * s
    else:
        y[..., :half], y[..., half:] = u * c - v * s, v * c + u * s
    return y


def turn_tolerance(x, y, interleaved, amplitude=1.0):
    """Half a bf16 step of the output; sine and cosine off by 2^-22 of the amplitude (their fp32 argument is within 2^-26 turns
    of the angle, and they are rounded), and three fp32 roundings of a product sum: 2^-21 of |u| + |v| in all."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    half = x.shape[-1] // 2
    m = np.empty_like(x)
    if interleaved:
        m[..., 0::2] = m[..., 1::2] = x[..., 0::2] + x[..., 1::2]
    else:
        m[..., :half] = m[..., half:] = x[..., :half] + x[..., half:]
    return 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * amplitude * m + 2.0 ** -133


# ---------------------------------------------------------------- the cache

def new_rows(x, L, weight=None, eps=0.0, positions=None, f=None, interleaved=True, amplitude=1.0):
    """Unrounded rows [n, L + R] of inputs x [n, L + R]; weight None: the latent part as it is; f None: the other as it is."""
    x = np.asarray(x, dtype=np.float64)
    c, r = x[:, :L], x[:, L:]
    if weight is not None:
        c = c / np.sqrt((c * c).mean(1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if f is not None:
        r = turn(r, positions, f, interleaved, amplitude)
    return np.concatenate([c, r], 1)


def rows_tolerance(x, y, L, interleaved=True, amplitude=1.0):
    """The latent part: half a bf16 step, an fp32 sum of L squares (each off by (L + 2) 2^-24 at most, half of it under the
    root), the root and three products: (L / 2 + 8) 2^-24 of the value.  The positional part: as turn_tolerance."""
    c = np.abs(y[:, :L]) * (2.0 ** -8 + (L / 2 + 8) * 2.0 ** -24) + 2.0 ** -133
    return np.concatenate([c, turn_tolerance(x[:, L:], y[:, L:], interleaved, amplitude)], 1)


# ---------------------------------------------------------------- attention

def decode(q, rows, L, scale):
    """(o, spread, shaken) of queries q [H, L + R] over rows [n, L + R]: spread is the same sum over |c|, shaken the largest sum
    of scale |q_i k_i| over the rows."""
    q, rows = np.asarray(q, dtype=np.float64), np.asarray(rows, dtype=np.float64)
    if len(rows) == 0:
        z = np.zeros((len(q), L))
        return z, z, np.zeros((len(q), 1))
    s = scale * (q @ rows.T)
    w = np.exp(s - s.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    shaken = scale * (np.abs(q) @ np.abs(rows).T).max(1)
    return w @ rows[:, :L], w @ np.abs(rows[:, :L]), shaken[:, None]


def attention_tolerance(o, spread, shaken, terms, score=0.0):
    """How far a kernel with bf16 output and weights and 32-bit sums may be off.

    bf16 output: 2^-8 |o|.  Weights rounded to bf16, off by 2^-8 of themselves at most, with a denominator that sums the rounded
    ones: 2^-8 sum_j p_j |c_j - o|, at most 2^-8 (spread + |o|).  A score is a sum of `terms` products in 32 bits, off by
    (terms + 8) 2^-24 of the sum of magnitudes with its scaling and shift, and by `score` where its operands were rounded: the
    error e enters numerator and denominator, 2 e of each term.  Exponentials, 32-bit sums and joins: 2^-18 of each term."""
    e = (terms + 8) * 2.0 ** -24 * shaken + score
    return 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -18) * (spread + np.abs(o)) + 2 * e * spread + 2.0 ** -133


def prefill(q, kv, k_rope, cu, scale, nope=128):
    """(o, spread, shaken) of q [T, H, nope + R], kv [T, H, nope + v], k_rope [T, R], causal over blocks cu[b] .. cu[b+1]."""
    q, kv, r = (np.asarray(a, dtype=np.float64) for a in (q, kv, k_rope))
    T, H = q.shape[:2]
    o, spread, shaken = np.zeros((T, H, kv.shape[2] - nope)), np.zeros((T, H, kv.shape[2] - nope)), np.zeros((T, H, 1))
    for a, b in zip(cu[:-1], cu[1:]):
        below = np.tril(np.ones((b - a, b - a), dtype=bool))
        for h in range(H):
            k = np.concatenate([kv[a:b, h, :nope], r[a:b]], 1)
            s = np.where(below, scale * (q[a:b, h] @ k.T), -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            v = kv[a:b, h, nope:]
            o[a:b, h], spread[a:b, h] = w @ v, w @ np.abs(v)
            shaken[a:b, h, 0] = np.where(below, scale * (np.abs(q[a:b, h]) @ np.abs(k).T), 0.0).max(1)
    return o, spread, shaken

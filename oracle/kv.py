"""Rotary positions, the paged key/value cache and attention over it, in f64.

Plain numpy from the definitions, one row, slot or query at a time; shares no
code with the library.  16-bit numbers arrive as f64 arrays of their exact
values; an 8-bit cache is a pair (codes as f64, f32 scales).
"""
from __future__ import annotations

import numpy as np

LARGEST = {"int8": 127.0, "e4m3": 448.0}


def rotate64(x, positions, freq, interleaved=False, magnitude=1.0, transpose=False):
    """x [T, heads, dim] turned pair by pair (2·len(freq) coordinates)."""
    x = np.array(x, np.float64)
    n = len(freq)
    for t, p in enumerate(positions):
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            angle = float(p) * float(freq[i])
            c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
            if transpose:
                s = -s
            xa, xb = x[t, :, a].copy(), x[t, :, b].copy()
            x[t, :, a], x[t, :, b] = c * xa - s * xb, s * xa + c * xb
    return x


def e4m3_values():
    """The non-negative e4m3 values: 4 exponent bits (bias 7), 3 of mantissa, no
    infinity, largest 448."""
    v = [m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
         for e in range(16) for m in range(8)]
    return np.array(v[:-1])          # the last code is the NaN


def nearest_code(x, kind):
    """x (scaled) to the nearest code's value, ties to even."""
    if kind == "int8":
        return np.clip(np.rint(x), -127, 127)
    grid = e4m3_values()
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    down, up = a - grid[lo], grid[hi] - a
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return np.copysign(grid[pick], x)


def quantise(x, kind):
    """Rows [..., dim] of f32 numbers -> (codes, scales): the scale and the quotient
    are f32 numbers, as the format defines them."""
    x = np.asarray(x, np.float32)
    scale = np.max(np.abs(x), -1) / np.float32(LARGEST[kind])
    bad = ~np.isfinite(x).all(-1)
    safe = np.where((scale > 0) & ~bad, scale, np.float32(1))
    q = np.where(((scale > 0) & ~bad)[..., None], x / safe[..., None], np.float32(0))
    return nearest_code(q.astype(np.float64), kind), np.where(bad, np.float32(np.nan), scale)


def key_index(slot, h, d, heads, page, dim):
    """Element of the key pages that holds coordinate d of a slot's head h."""
    return ((slot // page * heads + h) * page + slot % page) * dim + d


def value_index(slot, h, d, heads, page, dim, run):
    """Element of the value pages: runs of `run` places, coordinate by coordinate."""
    place = slot % page
    return ((slot // page * heads + h) * page + place - place % run) * dim + d * run + place % run


def attend64(q, k, v, new, length, causal=True, window=0, scale=None):
    """One sequence: q [new, q_heads, dim], k and v [length, heads, dim] ->
    (out, lse, weights [new, q_heads, length]); rows that see nothing: 0, −inf."""
    group = q.shape[1] // k.shape[1]
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    weights = np.zeros(q.shape[:2] + (length,))
    for i in range(new):
        p = length - new + i
        last = min(length, p + 1) if causal else length
        first = max(0, p - window + 1) if window else 0
        if last <= first:
            continue
        for h in range(q.shape[1]):
            s = scale * (k[first:last, h // group] @ q[i, h])
            m = s.max()
            w = np.exp(s - m)
            out[i, h] = w @ v[first:last, h // group] / w.sum()
            lse[i, h] = m + np.log(w.sum())
            weights[i, h, first:last] = w / w.sum()
    return out, lse, weights

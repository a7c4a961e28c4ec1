"""fp64 statements of the operators of a cache that grows token by token (test infrastructure, numpy only)."""
from __future__ import annotations

import math

import numpy as np

from . import token_ops


def visible(cached, pos, n, sinks, left, right):
    """[n, cached] truth values: which cached tokens the rows at positions pos .. pos + n - 1 see."""
    t = np.arange(cached)[None, :]
    p = pos + np.arange(n)[:, None]
    seen = np.ones((n, cached), dtype=bool)
    if right >= 0:
        seen &= t <= p + right
    if left >= 0:
        seen &= (t < sinks) | (t >= p - left)
    return seen


def attend_window(q, k, v, pos, sinks, left, right, scale):
    """One request: q [n, Hq, D], k, v [cached, Hkv, D], all that is cached.

    Returns out [n, Hq, D], lse [n, Hq], and for bounds of rounding errors the weighted magnitudes sum w |v| [n, Hq, D] and
    the largest scale * sum |q| |k| over the visible tokens [n, Hq].  Rows that see nothing: 0, -inf."""
    n, hq, d = q.shape
    cached, hkv = k.shape[:2]
    out, mag = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, size = np.full((n, hq), -math.inf), np.zeros((n, hq))
    seen = visible(cached, pos, n, sinks, left, right)
    some = seen.any(axis=1)
    used = seen.any(axis=0)                       # tokens that no row sees may hold anything
    if not some.any():
        return out, lse, mag, size
    k, v, seen = k[used], v[used], seen[:, used]
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        s = np.where(seen, scale * (q[:, h] @ kh.T), -math.inf)[some]
        top = s.max(axis=1)
        e = np.exp(s - top[:, None])
        total = e.sum(axis=1)
        w = e / total[:, None]
        out[some, h], mag[some, h] = w @ vh, w @ np.abs(vh)
        lse[some, h] = top + np.log(total)
        size[some, h] = np.where(seen[some], scale * (np.abs(q[some, h]) @ np.abs(kh).T), 0).max(axis=1)
    return out, lse, mag, size


def rope_axes_table(positions, freq, pair_axis, scale=1.0):
    """[rows, pairs, 2]; positions [axes][rows], pair_axis the axis of every pair."""
    rows = len(positions[0])
    out = np.empty((rows, len(freq), 2))
    for i, (f, a) in enumerate(zip(freq, pair_axis)):
        out[:, i:i + 1] = token_ops.rope_table(positions[a], [f], scale)
    return out


def rope_axes(x, positions, freq, pair_axis, interleaved=False, scale=1.0, inverse=False):
    """x [rows, heads, D] with the pairs of the first 2 * len(freq) dims rotated, each by the position of its axis."""
    y = np.array(x, dtype=np.float64)
    table = rope_axes_table(positions, freq, pair_axis)
    for i in range(len(freq)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(freq))
        z = (y[..., a] + 1j * y[..., b]) * np.conj(table[:, i, 0] + 1j * table[:, i, 1])[:, None] if inverse else \
            (y[..., a] + 1j * y[..., b]) * (table[:, i, 0] + 1j * table[:, i, 1])[:, None]
        z *= 1.0 / scale if inverse else scale
        y[..., a], y[..., b] = z.real, z.imag
    return y

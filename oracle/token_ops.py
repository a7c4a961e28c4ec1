"""fp64 statements of the token-eviction and rotary operators (test infrastructure, numpy only)."""
from __future__ import annotations

import math

import numpy as np


def prefix_weights(k, q, lse, group, scale, before=None, decay=0.0):
    """decay * before + sum over rows and the query heads of each KV head of exp(scale q.k - lse).

    k [m, Hkv, D] cached keys of one prefix, q [rows, Hq, D] the rows of its requests, lse [rows, Hq];
    group = Hq / Hkv.  Rows with an infinite lse add nothing.  Returns [Hkv, m]."""
    m, hkv, _ = k.shape
    out = np.zeros((hkv, m))
    if decay != 0.0:
        out += decay * np.asarray(before, dtype=np.float64)[:, :m]
    for j in range(hkv):
        for h in range(j * group, (j + 1) * group):
            live = ~np.isinf(lse[:, h])
            if live.any():
                s = scale * (k[:, j] @ q[live, h].T)
                with np.errstate(over="ignore", invalid="ignore"):
                    out[j] += np.exp(s - lse[live, h]).sum(axis=1)
    return out


def select_tokens(scores, keep, first=0, last=0):
    """Ascending indices of the kept tokens of one row: protected ends, then larger score, then lower index."""
    n = len(scores)
    first = min(first, n)
    last = min(last, n - first)
    s = [-math.inf if math.isnan(x) else float(x) for x in scores]
    order = sorted(range(n), key=lambda i: (not (i < first or i >= n - last), -s[i], i))
    return sorted(order[:keep])


def rope_frequencies(rot, base, scaling="none", factor=1.0, length=0, low=0.0, high=0.0):
    """Angle per position of pair i."""
    out = []
    for i in range(rot // 2):
        b = base
        if scaling == "ntk" and rot > 2:
            b = base * factor ** (rot / (rot - 2))
        f = b ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "yarn":
            at = [rot * math.log(length / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (high, low)]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            ramp = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = (f / factor) * ramp + f * (1 - ramp)
        elif scaling == "bands":
            keep = min(1.0, max(0.0, (length * f / (2 * math.pi) - low) / (high - low)))
            f = (f / factor) * (1 - keep) + f * keep
        out.append(f)
    return np.array(out)


def rope_table(positions, freq, scale=1.0):
    """[rows, pairs, 2] of (cos, sin) * scale; the angle is reduced in exact integer arithmetic of 2^-80 turns."""
    turn = [int(math.floor(f / (2 * math.pi) * 2.0 ** 52 + 0.5)) for f in freq]
    out = np.empty((len(positions), len(freq), 2))
    for r, p in enumerate(positions):
        for i, (t, f) in enumerate(zip(turn, freq)):
            # the part that 52 bits of a turn leave over is added as a small angle
            rest = f / (2 * math.pi) - t / 2.0 ** 52
            a = 2 * math.pi * (((int(p) * t) % (1 << 52)) / 2.0 ** 52 + int(p) * rest)
            out[r, i] = math.cos(a) * scale, math.sin(a) * scale
    return out


def rope(x, positions, freq, interleaved=False, scale=1.0, inverse=False):
    """x [rows, heads, D] with the pairs of the first 2 * len(freq) dims rotated."""
    y = np.array(x, dtype=np.float64)
    pairs = len(freq)
    table = rope_table(positions, freq)
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    if inverse:
        s, scale = -s, 1.0 / scale
    d = np.arange(pairs)
    i, j = (2 * d, 2 * d + 1) if interleaved else (d, d + pairs)
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i] = scale * (a * c - b * s)
    y[..., j] = scale * (b * c + a * s)
    return y

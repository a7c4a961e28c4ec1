"""The fp64 statements of windowed attention and of rotations with several axes, pinned by brute force and by the cases
where they must agree with simpler operators."""
import math

import numpy as np
import pytest

from oracle import growing_cache as gc
from oracle import token_ops as op


@pytest.mark.parametrize("sinks,left,right", [(0, -1, -1), (0, -1, 0), (2, 3, 0), (0, 0, 0), (3, 1, 4), (9, 2, -1), (0, 2, 1)])
@pytest.mark.parametrize("cached,pos,n", [(7, 0, 7), (7, 5, 4), (1, 0, 1), (0, 0, 2), (6, 11, 2), (9, 3, 1)])
def test_window_against_loops(sinks, left, right, cached, pos, n):
    rng = np.random.default_rng(cached * 31 + pos * 7 + n)
    q, k, v = rng.normal(size=(n, 4, 8)), rng.normal(size=(cached, 2, 8)), rng.normal(size=(cached, 2, 8))
    out, lse, mag, size = gc.attend_window(q, k, v, pos, sinks, left, right, 0.3)
    for a in range(n):
        p = pos + a
        seen = [t for t in range(cached) if (right < 0 or t <= p + right) and (left < 0 or t < sinks or t >= p - left)]
        for h in range(4):
            s = [0.3 * float(q[a, h] @ k[t, h // 2]) for t in seen]
            if not s:
                assert lse[a, h] == -math.inf and not out[a, h].any()
                continue
            total = sum(math.exp(x) for x in s)
            want = sum(math.exp(x) / total * v[t, h // 2] for x, t in zip(s, seen))
            np.testing.assert_allclose(out[a, h], want, rtol=1e-12, atol=1e-14)
            assert abs(lse[a, h] - math.log(total)) < 1e-12
            assert (mag[a, h] >= np.abs(out[a, h]) - 1e-14).all() and size[a, h] >= max(map(abs, s)) - 1e-14


def test_unseen_tokens_may_hold_anything():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(2, 2, 4)), rng.normal(size=(10, 1, 4)), rng.normal(size=(10, 1, 4))
    want = gc.attend_window(q, k, v, 8, 1, 2, 0, 1.0)
    k[2:5], v[2:5] = math.nan, math.inf
    for a, b in zip(gc.attend_window(q, k, v, 8, 1, 2, 0, 1.0), want):
        np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_axes(interleaved, inverse):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(5, 3, 12))
    freq = op.rope_frequencies(8, 10000.0)
    pos = [[3, 1, 4, 1, 5], [9, 2, 6, 5, 3]]
    one = gc.rope_axes(x, pos, freq, [0] * 4, interleaved, 1.5, inverse)
    np.testing.assert_allclose(one, op.rope(x, pos[0], freq, interleaved, 1.5, inverse), atol=1e-14)
    other = gc.rope_axes(x, pos, freq, [1] * 4, interleaved, 1.5, inverse)
    mixed = gc.rope_axes(x, pos, freq, [0, 1, 1, 0], interleaved, 1.5, inverse)
    for i, a in enumerate([0, 1, 1, 0]):
        dims = [2 * i, 2 * i + 1] if interleaved else [i, i + 4]
        np.testing.assert_array_equal(mixed[..., dims], (other if a else one)[..., dims])
    np.testing.assert_array_equal(mixed[..., 8:], x[..., 8:])

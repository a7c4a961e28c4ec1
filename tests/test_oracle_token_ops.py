"""Pins of oracle.token_ops (fp64, CPU)."""
import math

import numpy as np
import pytest

from oracle import token_ops as op


def test_weights_are_the_attention_matrix_summed_over_rows():
    rng = np.random.default_rng(1)
    m, hkv, group, d, rows = 5, 2, 3, 8, 4
    k, q = rng.normal(size=(m, hkv, d)), rng.normal(size=(rows, hkv * group, d))
    s = np.array([[[0.3 * float(q[r, h] @ k[t, h // group]) for t in range(m)] for h in range(hkv * group)]
                  for r in range(rows)])
    lse = np.log(np.exp(s).sum(-1))
    w = op.prefix_weights(k, q, lse, group, 0.3)
    ref = np.zeros((hkv, m))
    for r in range(rows):
        for h in range(hkv * group):
            ref[h // group] += np.exp(s[r, h]) / np.exp(s[r, h]).sum()
    np.testing.assert_allclose(w, ref, rtol=1e-12)
    np.testing.assert_allclose(w.sum(1), rows * group)          # every row and head hands out weight 1
    lse[1] = np.inf
    lse[2, 0] = -np.inf
    before = rng.normal(size=(hkv, m + 2))
    w2 = op.prefix_weights(k, q, lse, group, 0.3, before, 0.5)
    np.testing.assert_allclose((w2 - 0.5 * before[:, :m]).sum(1), [2 * group + group - 1, 3 * group])


def test_select_by_hand():
    nan, inf = math.nan, math.inf
    assert op.select_tokens([1, 3, 2, 3, 3], 2) == [1, 3]                     # ties: lower index
    assert op.select_tokens([1, 3, 2, 3, 3], 3, first=1, last=1) == [0, 1, 4]
    assert op.select_tokens([nan, -inf, 0.0, -0.0], 3) == [0, 2, 3]           # NaN ranks as -inf, -0 as 0
    assert op.select_tokens([nan, -inf], 1) == [0]
    assert op.select_tokens([inf, 5, inf], 2, last=1) == [0, 2]
    assert op.select_tokens([1, 2, 3], 3, first=9, last=9) == [0, 1, 2]
    assert op.select_tokens([1, 2, 3], 0) == []


def test_rope_turns_and_differences():
    f = op.rope_frequencies(8, 10000.0)
    np.testing.assert_allclose(f, [1, 0.1, 0.01, 0.001])
    quarter = np.array([math.pi / 2])
    x = np.array([[[1.0, 2.0, 5.0, 7.0]]])
    np.testing.assert_allclose(op.rope(x, [1], quarter)[0, 0], [-2, 1, 5, 7], atol=1e-12)
    np.testing.assert_allclose(op.rope(np.arange(4.0).reshape(1, 1, 4), [3], [math.pi / 2, 0.0], interleaved=True)[0, 0],
                               [1, 0, 2, 3], atol=1e-12)
    rng = np.random.default_rng(2)
    a, b = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    far = float((op.rope(a, [1000007], f) * op.rope(b, [1000003], f)).sum())
    near = float((op.rope(a, [4], f) * b).sum())
    assert abs(far - near) < 1e-9
    back = op.rope(op.rope(a, [777], f, scale=1.25), [777], f, scale=1.25, inverse=True)
    np.testing.assert_allclose(back, a, rtol=1e-12)
    t = op.rope_table([5], f, 2.0)
    np.testing.assert_allclose(t[0, :, 0], 2 * np.cos(5 * f))
    np.testing.assert_allclose(t[0, :, 1], 2 * np.sin(5 * f))


@pytest.mark.parametrize("rot", [2, 64, 128])
def test_frequency_rules_at_their_ends(rot):
    plain = op.rope_frequencies(rot, 10000.0)
    np.testing.assert_allclose(op.rope_frequencies(rot, 10000.0, "linear", 4.0), plain / 4)
    ntk = op.rope_frequencies(rot, 10000.0, "ntk", 8.0)
    assert ntk[0] == 1.0
    if rot > 2:
        np.testing.assert_allclose(ntk[-1], plain[-1] / 8)                    # the slowest pair is interpolated fully
    for rule in ("yarn", "bands"):
        f = op.rope_frequencies(rot, 10000.0, rule, 16.0, 4096, 1.0, 32.0)
        assert f[0] == plain[0] and (f <= plain).all() and (f >= plain / 16 * (1 - 1e-12)).all()
        if rot > 2:
            np.testing.assert_allclose(f[-1], plain[-1] / 16)

"""GPU parity of rotary positions with several axes against the fp64 oracle, and bit for bit with the calls of one axis.

Tolerance as for the rotary calls of one axis: cosine and sine off by at most E = 1.5e-7, four fp32 roundings of at most
(|a| + |b|) scale, one rounding to the type of half a step."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from oracle import growing_cache as gc
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
E = 1.5e-7


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def f64(t):
    return workloads.to_f64(t)


def rows_of(n, heads, d, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, heads + pad, d), generator=g, device="cuda").to(dtype)[:, :heads]


def check(got, x, pos, freq, axis, interleaved, scale, inverse, dtype):
    ref = gc.rope_axes(f64(x), pos, freq, axis, interleaved, scale, inverse)
    pairs, ax = len(freq), np.abs(f64(x))
    size = np.zeros_like(ax)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        size[..., a] = size[..., b] = ax[..., a] + ax[..., b]
    inner = abs(1 / scale if inverse else scale) * size * (E + 4 * 2.0 ** -24)
    err = np.abs(f64(got) - ref)
    assert (err <= inner + (np.abs(ref) + inner) * torch.finfo(dtype).eps / 2).all(), err.max()
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,rot,axes", [(7, 1, 128, 128, 3), (4, 4, 64, 64, 2), (2, 1, 128, 32, 4), (3, 3, 96, 20, 3),
                                               (6, 2, 128, 2, 1), (2, 2, 256, 256, 3), (28, 4, 128, 108, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows(dtype, hq, hkv, d, rot, axes, interleaved):
    bc = binding.BiCache(1, hq, hkv, d, 8, dtype, 16, 1)
    n = 23
    q, k = rows_of(n, hq, d, dtype, 1, 1), rows_of(n, hkv, d, dtype, 2, 2)
    freq = binding.rope_frequencies(rot, 10000.0)
    rng = np.random.default_rng(rot)
    axis = rng.integers(0, axes, rot // 2).tolist()
    p = rng.integers(-1000, 1 << 20, (axes, n))
    pos = torch.tensor(p, dtype=torch.int32, device="cuda")
    r = binding.Rotation(freq, interleaved, 1.25, axis, axes)
    qo, ko = torch.full_like(rows_of(n, hq, d, dtype, 3, 1), 7), torch.empty_like(k)
    bc.rope_axes(r, pos, q, qo, k, ko)
    check(qo, q, p.tolist(), freq, axis, interleaved, 1.25, False, dtype)
    check(ko, k, p.tolist(), freq, axis, interleaved, 1.25, False, dtype)
    q2 = q.clone()
    bc.rope_axes(r, pos, q2, q2)                               # in place, no keys
    assert torch.equal(q2, qo)
    back = torch.empty_like(k)
    bc.rope_axes(r, pos, None, None, ko, back, inverse=True)
    check(back, ko, p.tolist(), freq, axis, interleaved, 1.25, True, dtype)
    # every axis by itself is the rotation by one axis
    for a in range(axes):
        alone = binding.Rotation(freq, interleaved, 1.25, [a] * (rot // 2), axes)
        want = torch.empty_like(q)
        bc.rope_axes(alone, pos, q, qo)
        bc.rope(freq, q, want, positions=pos[a], interleaved=interleaved, attention_scale=1.25)
        assert torch.equal(qo, want)


@pytest.mark.parametrize("rows", [0, 1, 3, 64, 8 * 148 + 1, 5000])
def test_row_counts_and_rows_behind_the_last(rows):
    bc = binding.BiCache(1, 14, 2, 128, 8, torch.bfloat16, 16, 1)
    freq, axis = binding.rope_frequencies(128, 10000.0), [i % 3 for i in range(64)]
    q = rows_of(rows + 2, 14, 128, torch.bfloat16, 5)
    out = torch.full_like(q, 3)
    p = np.random.default_rng(rows).integers(0, 40000, (3, rows + 5))
    pos = torch.tensor(p, dtype=torch.int32, device="cuda")
    bc.rope_axes(binding.Rotation(freq, pair_axis=axis, num_axes=3), pos[:, :rows], q[:rows], out[:rows])
    assert (out[rows:] == 3).all()
    some = list(range(0, rows, max(1, rows // 50)))
    if some:
        check(out[some], q[some], p[:, some].tolist(), freq, axis, False, 1.0, False, torch.bfloat16)


@pytest.mark.parametrize("rot,rows", [(2, 9), (64, 1), (128, 700), (256, 33), (6, 100)])
def test_table(rot, rows):
    bc = binding.BiCache(1, 2, 1, 128, 8, torch.bfloat16, 16, 1)
    freq, axis = binding.rope_frequencies(rot, 10000.0), [i % 3 for i in range(rot // 2)]
    p = np.random.default_rng(rot).integers(-5, 1 << 21, (3, rows))
    pos = torch.tensor(p, dtype=torch.int32, device="cuda")
    table = torch.empty((rows, rot // 2, 2), device="cuda")
    bc.rope_axes_table(binding.Rotation(freq, attention_scale=1.5, pair_axis=axis, num_axes=3), pos, table)
    err = np.abs(f64(table) - gc.rope_axes_table(p.tolist(), freq, axis, 1.5))
    # the frequency itself is a double: 2^-53 of 2^21 radians is 2.4e-10
    assert (err <= 1.5 * (E + 2 * 2.0 ** -24 + 1e-9)).all(), err.max()


def test_the_table_rotates_projected_keys():
    """project_prefix_layer with the table of several axes stores what rope_axes makes of the unrotated keys."""
    m, dm = 50, 64
    bc = binding.BiCache(1, 2, 1, 128, 8, torch.bfloat16, 64, 1)
    h, wk, wv = (rows_of(*s, torch.bfloat16, i) for i, s in enumerate(((1, m, dm), (1, 128, dm), (1, 128, dm))))
    freq, axis = binding.rope_frequencies(128, 10000.0), [i // 22 for i in range(64)]
    pos = torch.randint(0, 5000, (3, m), generator=torch.Generator().manual_seed(0), dtype=torch.int32).cuda()
    r = binding.Rotation(freq, pair_axis=axis, num_axes=3)
    table = torch.empty((m, 64, 2), device="cuda")
    bc.rope_axes_table(r, pos, table)
    pid = bc.reserve_prefix(1, m)[0]
    bc.project_prefix_layer(pid, 0, h[0], wk[0], wv[0], rope=table)
    k, v = torch.empty((m, 1, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((m, 1, 128), dtype=torch.bfloat16, device="cuda")
    bc.read_prefix_layer(pid, 0, k, v)
    assert bc.device_status() == 0
    plain = f64(h[0]) @ f64(wk[0]).T
    ref = gc.rope_axes(plain[:, None, :], pos.tolist(), freq, axis)
    size = np.abs(f64(h[0])) @ np.abs(f64(wk[0])).T            # 64 products, added in fp32, then the rotation
    inner = (size + np.roll(size, 64, axis=1))[:, None, :] * (64 * 2.0 ** -23 + E + 2.0 ** -22)
    assert (np.abs(f64(k) - ref) <= inner + (np.abs(ref) + inner) * 2.0 ** -8).all()

"""A growing cache whose layers differ: pools of different sizes, prefixes that own the deeper layers only, page lists that
are not the same in every layer (after evictions), tokens that several rows of one call become, and calls on a stream of
their own."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from oracle import growing_cache as gc
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def f64(t):
    return workloads.to_f64(t)


def randn(shape, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("hq,hkv,d,dtype", [(14, 2, 128, torch.bfloat16), (4, 4, 64, torch.float32)])
def test_layers_that_differ(hq, hkv, d, dtype, seed):
    rng = np.random.default_rng(seed)
    caps = [70, 90, 80]
    bc = binding.BiCache(3, hq, hkv, d, 90, dtype, 900, 8, layer_pages=caps, free_order=rng.permutation(90) if seed % 2 else None)
    bc.k_pool.fill_(255)
    bc.v_pool.fill_(255)
    live = {}                                                  # id: length, first layer, K and V per layer
    stream = torch.cuda.Stream()
    for step in range(14):
        m, first = int(rng.integers(1, 400)), int(rng.integers(0, 3))
        pid = bc.reserve_prefix(1000 + step, m, first)[0]      # evicts the oldest ones
        for old in list(live):
            try:
                bc.prefix_pages(old)
            except binding.BiCacheError:
                del live[old]
        live[pid] = (m, first, {l: (randn((m, hkv, d), 100 * step + l, dtype), randn((m, hkv, d), 100 * step + 50 + l, dtype)) for l in range(first, 3)})
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for l in range(first, 3):
                k, v = live[pid][2][l]
                cut = int(rng.integers(0, m + 1))
                bc.append_tokens(l, [pid, pid], [cut, 0], [cut, 0], [m - cut, cut], k, v)
            for l in range(3):
                ids = [i for i, (_, f, _) in live.items() if f <= l]
                if not ids:
                    continue
                n = [int(rng.integers(1, 40)) for _ in ids]
                pos = [int(rng.integers(0, live[i][0] + 5)) for i in ids]
                cached = [int(rng.integers(0, live[i][0] + 1)) for i in ids]
                off = (np.cumsum(n) - n).tolist()
                q = randn((sum(n), hq, d), step, dtype)
                out, lse = torch.empty_like(q), torch.empty((sum(n), hq), device="cuda")
                bc.attend_window(l, ids, cached, pos, off, n, q, out, lse, 3, 90, 7)
                kb, vb = (torch.empty((live[ids[0]][0], hkv, d), dtype=dtype, device="cuda") for _ in range(2))
                bc.read_tokens(l, ids[:1], [0], [0], [live[ids[0]][0]], kb, vb)
                stream.synchronize()
                assert torch.equal(kb, live[ids[0]][2][l][0]) and torch.equal(vb, live[ids[0]][2][l][1])
                for i, o, c, p, c_len in zip(ids, off, n, pos, cached):
                    k, v = live[i][2][l]
                    ref, rl, mag, size = gc.attend_window(f64(q[o:o + c]), f64(k[:c_len]), f64(v[:c_len]), p, 3, 90, 7, d ** -0.5)
                    steps = (c_len / 16 + 64) * 2.0 ** -23     # bounds as in test_gpu_attend_window.py
                    e = (d + 8) * 2.0 ** -23 * size + 2.0 ** -20
                    tol = mag * ((2.0 ** -8 if dtype == torch.bfloat16 else 0) + 2 * e + steps)[..., None]
                    assert (np.abs(f64(out[o:o + c]) - ref) <= tol + (np.abs(ref) + tol) * torch.finfo(dtype).eps / 2).all()
                    none, got = np.isneginf(rl), f64(lse[o:o + c])
                    assert (np.isneginf(got) == none).all()
                    assert (np.abs(got[~none] - rl[~none]) <= (e + steps + 2.0 ** -22 * (np.abs(rl) + size + 8))[~none]).all()
    assert bc.device_status() == 0 and len(live) > 1


@pytest.mark.parametrize("dtype,d,rot", [(torch.bfloat16, 128, 128), (torch.bfloat16, 128, 36), (torch.float32, 64, 64)])
def test_rows_that_become_tokens_of_several_prefixes(dtype, d, rot):
    """Keys and values alone: each copy is rotated to its own place."""
    hkv, n = 2, 45
    bc = binding.BiCache(1, 4, hkv, d, 40, dtype, 64, 4)
    ids = [bc.reserve_prefix(i, 200)[0] for i in range(3)]
    k, v = randn((n, hkv, d), 1, dtype), randn((n, hkv, d), 2, dtype)
    freq = binding.rope_frequencies(rot, 10000.0)
    at = [0, 77, 150]
    bc.append_tokens(0, ids, at, [0, 0, 5], [n, n, n - 5], k, v, rotation=binding.Rotation(freq))
    for i, t, o, c in zip(ids, at, [0, 0, 5], [n, n, n - 5]):
        kb, vb, want = (torch.empty((c, hkv, d), dtype=dtype, device="cuda") for _ in range(3))
        bc.read_tokens(0, [i], [t], [0], [c], kb, vb)
        bc.rope(freq, None, None, k[o:o + c], want, position0=t)
        assert torch.equal(vb, v[o:o + c])
        size = (f64(k[o:o + c]) ** 2).sum(-1, keepdims=True) ** 0.5
        err = np.abs(f64(kb) - f64(want))                      # two fp32 forms of one rotation, each rounded once
        assert (err <= np.abs(f64(want)) * torch.finfo(dtype).eps + size * 6 * 2.0 ** -24).all()

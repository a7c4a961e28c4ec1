"""Attention over a cache that was thinned out to the tokens attended to most, and appended to since, at the bounds of the
attention tests (test_gpu_attend_window.py): a dropped or repeated token of ordinary weight does not pass."""
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


def bounds(d, count, mag, size, rl, ref, dtype):
    """Of the output and of its log-sum-exp over `count` cached tokens."""
    steps = (count / 16 + 64) * 2.0 ** -23
    e = (d + 8) * 2.0 ** -23 * size + 2.0 ** -20
    tol = mag * ((2.0 ** -8 if dtype == torch.bfloat16 else 0) + 2 * e + steps)[..., None]
    return tol + (np.abs(ref) + tol) * torch.finfo(dtype).eps / 2, e + steps + 2.0 ** -22 * (np.abs(rl) + size + 8)


@pytest.mark.parametrize("n", [5, 1])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(14, 2, 128, torch.bfloat16), (4, 4, 128, torch.bfloat16), (4, 4, 64, torch.float32)])
def test_thinned_out_and_appended_to(hq, hkv, d, dtype, n):
    m, keep, more = 611, 300, 17
    bc = binding.BiCache(2, hq, hkv, d, 120, dtype, m, 2, free_order=np.random.default_rng(2).permutation(120))
    bc.k_pool.fill_(255)
    bc.v_pool.fill_(255)
    k, v, q = randn((m, hkv, d), 1, dtype), randn((m, hkv, d), 2, dtype), randn((n, hq, d), 3, dtype)
    whole, kept = bc.reserve_prefix(1, m)[0], bc.reserve_prefix(2, keep)[0]
    grown = bc.reserve_prefix(3, keep + 40)[0]
    bc.append_tokens(1, [whole], [0], [0], [m], k, v)
    out, lse = torch.empty_like(q), torch.empty((n, hq), device="cuda")
    scores = torch.empty((hkv, m), device="cuda")
    bc.attend_window(1, [whole], [m], [m], [0], [n], q, out, lse)
    bc.prefix_weights(1, [whole], [0], [n], q, lse, scores, [0])
    idx = torch.empty((1, hkv, keep), dtype=torch.int32, device="cuda")
    bc.select_tokens(scores, keep, idx[0], protect_first=4, protect_last=16)
    bc.compact_prefix(whole, kept, idx, first_layer=1)
    # what the indices name, by the rows themselves: per head its own tokens
    at = idx[0].long().t()[:, :, None].expand(keep, hkv, d)
    k1, v1 = torch.gather(k, 0, at), torch.gather(v, 0, at)
    kb, vb = torch.empty_like(k1), torch.empty_like(v1)
    bc.read_tokens(1, [kept], [0], [0], [keep], kb, vb)
    assert torch.equal(kb, k1) and torch.equal(vb, v1)
    # a longer prefix takes them over and grows
    k2, v2 = randn((more, hkv, d), 4, dtype), randn((more, hkv, d), 5, dtype)
    bc.append_tokens(1, [grown, grown], [0, keep], [0, keep], [keep, more], torch.cat([kb, k2]), torch.cat([vb, v2]))
    kk, vv, held = f64(torch.cat([k1, k2])), f64(torch.cat([v1, v2])), keep + more
    for window in ((4, -1, -1), (4, 200, 0)):
        bc.attend_window(1, [grown], [held], [held - n], [0], [n], q, out, lse, *window)
        assert bc.device_status() == 0
        ref, rl, mag, size = gc.attend_window(f64(q), kk, vv, held - n, *window, d ** -0.5)
        tol, lse_tol = bounds(d, held, mag, size, rl, ref, dtype)
        assert (np.abs(f64(out) - ref) <= tol).all() and (np.abs(f64(lse) - rl) <= lse_tol).all()
        if window[1] >= 0:
            continue
        # The bounds tell the definition without a token of middling weight, and with it twice, from the right one: a form
        # that is off by up to the bound itself, and makes that mistake, is still off by more than it somewhere.
        weight = np.exp(d ** -0.5 * (kk[:, 0] @ f64(q)[0, 0]))
        token = np.argsort(weight)[held // 2]
        for rows in (np.delete(np.arange(held), token), np.insert(np.arange(held), token, token)):
            wrong, wl, _, _ = gc.attend_window(f64(q), kk[rows], vv[rows], len(rows) - n, *window, d ** -0.5)
            assert (np.abs(wl - rl) > 2 * lse_tol).any()

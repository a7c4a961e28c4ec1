"""A run of the calls on a growing cache as decoding makes them: a prompt, blocks and single tokens are appended layer by
layer, attended to under a window, the cache is thinned out and decoding goes on; directly and captured into graphs."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from oracle import growing_cache as gc
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def f64(t):
    return workloads.to_f64(t)


def randn(shape, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(14, 2, 128, torch.bfloat16), (4, 4, 64, torch.float32)])
def test_decoding(hq, hkv, d, dtype):
    """Two requests, two layers: prompts of odd lengths, then a block of 8 and single tokens."""
    L, caps = 2, [700, 333]
    bc = binding.BiCache(L, hq, hkv, d, 160, dtype, 1100, 2)
    bc.k_pool.fill_(255)
    bc.v_pool.fill_(255)
    ids = [bc.reserve_prefix(i + 1, c)[0] for i, c in enumerate(caps)]
    rot = binding.Rotation(binding.rope_frequencies(d, 10000.0))
    freq, axis = binding.rope_frequencies(d, 10000.0), [0] * (d // 2)
    keys = [[np.zeros((0, hkv, d)) for _ in caps] for _ in range(L)]           # what the cache has to hold
    values = [[np.zeros((0, hkv, d)) for _ in caps] for _ in range(L)]
    held = [0, 0]
    sinks, left = 4, 150
    for step, lens in enumerate([(601, 290), (8, 8), (1, 1), (1, 0), (1, 3)]):
        off, rows = [0, lens[0]], sum(lens)
        for layer in range(L):
            q, k, v = (randn((rows, h, d), 100 * step + 10 * layer + i, dtype) for i, h in enumerate((hq, hkv, hkv)))
            bc.append_tokens(layer, ids, held, off, lens, k, v, q, q, rot)
            out, lse = torch.empty_like(q), torch.empty((rows, hq), device="cuda")
            cached = [h + n for h, n in zip(held, lens)]
            kb, vb = torch.empty_like(k), torch.empty_like(v)
            bc.read_tokens(layer, ids, held, off, lens, kb, vb)
            bc.attend_window(layer, ids, cached, held, off, lens, q, out, lse, sinks=sinks, left=left, right=7)
            assert bc.device_status() == 0
            for i, n in enumerate(lens):
                if n == 0:
                    continue
                r = slice(off[i], off[i] + n)
                want = gc.rope_axes(f64(k[r]), [list(range(held[i], held[i] + n))], freq, axis)
                np.testing.assert_allclose(f64(kb[r]), want, atol=2e-6 + np.abs(want).max() * torch.finfo(dtype).eps / 2)
                keys[layer][i] = np.concatenate([keys[layer][i], f64(kb[r])])
                values[layer][i] = np.concatenate([values[layer][i], f64(v[r])])
                ref, rl, mag, size = gc.attend_window(f64(q[r]), keys[layer][i], values[layer][i], held[i], sinks, left, 7, d ** -0.5)
                e = (d + 8) * 2.0 ** -23 * size + 2.0 ** -20
                tol = mag * ((2.0 ** -8 if dtype == torch.bfloat16 else 0) + 2 * e + 110 * 2.0 ** -23)[..., None]
                assert (np.abs(f64(out[r]) - ref) <= tol + (np.abs(ref) + tol) * torch.finfo(dtype).eps / 2).all()
                assert (np.abs(f64(lse[r]) - rl) <= e + 110 * 2.0 ** -23 + 2.0 ** -22 * (np.abs(rl) + size + 8)).all()
        held = cached
    # thin out the first request's cache to the tokens that the last rows attend to most, and attend over what is left
    m, keep = held[0], 300
    whole = bc.reserve_prefix(9, m)[0]                         # the weights call takes whole prefixes
    for layer in range(L):
        k, v = (torch.tensor(x, dtype=torch.float32, device="cuda").to(dtype) for x in (keys[layer][0], values[layer][0]))
        bc.append_tokens(layer, [whole], [0], [0], [m], k, v)
    q = randn((5, hq, d), 999, dtype)
    lse, out = torch.empty((5, hq), device="cuda"), torch.empty_like(q)
    scores = torch.empty((hkv, m), device="cuda")
    bc.attend_window(0, [whole], [m], [m], [0], [5], q, out, lse)
    bc.prefix_weights(0, [whole], [0], [5], q, lse, scores, [0])
    np.testing.assert_allclose(f64(scores).sum(1), 5 * hq // hkv, rtol=1e-3)  # every row and head hands out weight 1
    idx = torch.empty((1, hkv, keep), dtype=torch.int32, device="cuda")
    bc.select_tokens(scores, keep, idx[0], protect_first=4, protect_last=16)
    short = bc.reserve_prefix(10, keep + 20)[0]
    kept = bc.reserve_prefix(11, keep)[0]
    bc.compact_prefix(whole, kept, idx)
    k, v = torch.empty((keep, hkv, d), dtype=dtype, device="cuda"), torch.empty((keep, hkv, d), dtype=dtype, device="cuda")
    bc.read_tokens(0, [kept], [0], [0], [keep], k, v)
    bc.append_tokens(0, [short], [0], [0], [keep], k, v)       # with room to go on
    bc.attend_window(0, [short], [keep], [keep], [0], [5], q, out, lse, sinks=4, left=-1)
    ref, rl, mag, size = gc.attend_window(f64(q), f64(k), f64(v), keep, 4, -1, -1, d ** -0.5)
    assert bc.device_status() == 0
    assert (np.abs(f64(out) - ref) <= mag * 0.01 + np.abs(ref) * torch.finfo(dtype).eps).all()


@pytest.mark.parametrize("dtype,hq,hkv,d,pages", [(torch.bfloat16, 32, 32, 128, 40000), (torch.float32, 32, 32, 64, 40000)])
def test_pages_beyond_32_bits_of_bytes(dtype, hq, hkv, d, pages):
    """The last pages of pools of 5.2 GB each."""
    m, n = 300, 40
    for order in (list(range(pages))[::-1], list(range(pages - 19, pages)) + list(range(pages - 19))):     # listed, consecutive
        bc = binding.BiCache(1, hq, hkv, d, pages, dtype, 64, 1, free_order=order)
        pid, _, own = bc.reserve_prefix(1, m)
        assert min(own) >= pages - 19
        k, v, q = randn((m, hkv, d), 1, dtype), randn((m, hkv, d), 2, dtype), randn((n, hq, d), 3, dtype)
        kb, vb, out = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
        bc.append_tokens(0, [pid], [0], [0], [m], k, v)
        bc.read_tokens(0, [pid], [0], [0], [m], kb, vb)
        assert torch.equal(kb, k) and torch.equal(vb, v)
        bc.attend_window(0, [pid], [m], [m - n], [0], [n], q, out, None, 4, 100, 0)
        assert bc.device_status() == 0
        ref, _, mag, size = gc.attend_window(f64(q), f64(k), f64(v), m - n, 4, 100, 0, d ** -0.5)
        e = ((d + 8) * 2.0 ** -23 * size + 2.0 ** -20)[..., None]
        tol = mag * ((2.0 ** -8 if dtype == torch.bfloat16 else 0) + 2 * e + 90 * 2.0 ** -23)
        assert (np.abs(f64(out) - ref) <= tol + (np.abs(ref) + tol) * torch.finfo(dtype).eps / 2).all()
        bc.close()


FIRST = """
import torch
from paper_2606_07571_b200 import binding

def randn(*shape, dtype):
    return torch.randn(shape, device="cuda").to(dtype)

for dtype, d, rot in ((torch.bfloat16, 128, 128), (torch.float32, 64, 20)):
    bc = binding.BiCache(1, 4, 2, d, 1400, dtype, 16, 1)
    long, _, _ = bc.reserve_prefix(1, 20000)
    short, _, _ = bc.reserve_prefix(2, 500)
    k, v, q = randn(20500, 2, d, dtype=dtype), randn(20500, 2, d, dtype=dtype), randn(20500, 4, d, dtype=dtype)
    r = binding.Rotation(binding.rope_frequencies(rot, 10000.0), pair_axis=[i % 2 for i in range(rot // 2)], num_axes=2)
    pos = torch.arange(41000, dtype=torch.int32, device="cuda").view(2, 20500)
    batch = ([long, short], [0, 0], [0, 20000], [20000, 500])

    def outputs():
        return dict(q=torch.zeros_like(q), q2=torch.zeros_like(q), out=torch.zeros_like(q), one=torch.zeros_like(q[:1]),
                    lse=torch.zeros((20500, 4), device="cuda"), gk=torch.zeros_like(k), gv=torch.zeros_like(v),
                    table=torch.zeros((20500, rot // 2, 2), device="cuda"))

    def calls(o):
        bc.append_tokens(0, *batch, k, v, q, o["q"], r, pos)
        bc.read_tokens(0, *batch, o["gk"], o["gv"])
        bc.attend_window(0, batch[0], [20000, 500], [0, 0], batch[2], batch[3], o["q"], o["out"], o["lse"], 4, 900, 0)
        bc.attend_window(0, [long], [20000], [19999], [0], [1], q[:1], o["one"])
        bc.rope_axes(r, pos, q, o["q2"])
        bc.rope_axes_table(r, pos, o["table"])

    captured, direct = outputs(), outputs()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls(captured)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    calls(direct)
    assert bc.device_status() == 0
    for name in captured:
        assert torch.equal(captured[name], direct[name]) and captured[name].abs().sum() > 0, name
print("same")
"""


def test_a_process_may_begin_with_a_capture():
    run = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "same", run.stderr[-3000:]


def test_two_graphs_that_share_the_workspace():
    bc = binding.BiCache(1, 14, 2, 128, 2600, torch.bfloat16, 16, 2)
    parts = []
    for key, m, n in ((1, 20000, 2), (2, 15000, 5)):           # keys split into ranges: partial results in the workspace
        k, v, q = randn((m, 2, 128), key, torch.bfloat16), randn((m, 2, 128), key + 10, torch.bfloat16), randn((n, 14, 128), key + 20, torch.bfloat16)
        pid = bc.reserve_prefix(key, m)[0]
        bc.append_tokens(0, [pid], [0], [0], [m], k, v)
        out, want = torch.zeros_like(q), torch.zeros_like(q)

        def call(out, pid=pid, m=m, n=n, q=q):
            bc.attend_window(0, [pid], [m], [m - n], [0], [n], q, out, right=0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        launches = bc.launch_count()
        with torch.cuda.graph(graph):
            call(out)
        assert bc.launch_count() == launches + 2
        parts.append((graph, call, out, want))
    for i in (0, 1, 1, 0, 1):
        parts[i][0].replay()
    for _, call, _, want in parts:
        call(want)
    assert bc.device_status() == 0
    for _, _, out, want in parts:
        assert torch.equal(out, want) and out.abs().sum() > 0

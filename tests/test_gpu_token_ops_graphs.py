"""Token-eviction and rotary calls in CUDA graphs: captured as a process's first launches of these kernels, and as two
graphs of one context that share its workspace and follow one another."""
import os
import subprocess
import sys

import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST = """
import torch
from paper_2606_07571_b200 import binding

def randn(*shape, dtype):
    return torch.randn(shape, device="cuda").to(dtype)

for dtype, d, rot in ((torch.bfloat16, 128, 128), (torch.float32, 64, 20)):
    m, n, keep = 40, 1600, 8                       # as many rows as are split into ranges
    bc = binding.BiCache(1, 4, 2, d, 8, dtype, 16, 1)
    k = randn(1, m, 2, d, dtype=dtype)
    src, _, _ = bc.put_prefix(1, k, -k)
    dst, _, _ = bc.reserve_prefix(2, keep)
    q, own = randn(n, 4, d, dtype=dtype), randn(n, 2, d, dtype=dtype)
    lse = torch.full((n, 4), 9.0, device="cuda")
    freq = binding.rope_frequencies(rot, 10000.0)

    def outputs():
        return dict(q=torch.zeros_like(q), k=torch.zeros_like(own), table=torch.zeros((m, rot // 2, 2), device="cuda"),
                    w=torch.zeros((2, m), device="cuda"), idx=torch.zeros((1, 2, keep), dtype=torch.int32, device="cuda"),
                    gk=torch.zeros((keep, 2, d), dtype=dtype, device="cuda"), gv=torch.zeros((keep, 2, d), dtype=dtype, device="cuda"))

    def calls(o):
        bc.rope(freq, q, o["q"], own, o["k"], position0=5)
        bc.rope_table(freq, o["table"])
        bc.prefix_weights(0, [src], [0], [n], q, lse, o["w"], [0])
        bc.select_tokens(o["w"], keep, o["idx"][0], 1, 1)
        bc.compact_prefix(src, dst, o["idx"])
        bc.read_prefix_layer(dst, 0, o["gk"], o["gv"])

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


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def test_a_process_may_begin_with_a_capture():
    run = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "same", run.stderr[-3000:]


def test_two_graphs_that_share_the_workspace():
    bc = binding.BiCache(1, 14, 2, 128, 8, torch.bfloat16, 16, 2)
    g = torch.Generator(device="cuda").manual_seed(1)
    parts = []
    for key, m, n in ((1, 40, 1600), (2, 30, 1200)):              # rows split into ranges: partial sums in the workspace
        k = torch.randn((1, m, 2, 128), generator=g, device="cuda").bfloat16()
        pid, _, _ = bc.put_prefix(key, k, k)
        q = torch.randn((n, 14, 128), generator=g, device="cuda").bfloat16()
        lse = torch.full((n, 14), 6.0, device="cuda")
        scores, want = torch.zeros((2, m), device="cuda"), torch.zeros((2, m), device="cuda")

        def call(out, pid=pid, n=n, q=q, lse=lse):
            bc.prefix_weights(0, [pid], [0], [n], q, lse, out, [0], scores_in=out, decay=0.5)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        launches = bc.launch_count()
        with torch.cuda.graph(graph):
            call(scores)
        assert bc.launch_count() == launches + 2
        parts.append((graph, call, scores, want))
    order = [0, 1, 1, 0, 1]
    for i in order:
        parts[i][0].replay()
    for i in order:
        parts[i][1](parts[i][3])
    assert bc.device_status() == 0
    for _, _, scores, want in parts:
        assert torch.equal(scores, want) and scores.abs().sum() > 0

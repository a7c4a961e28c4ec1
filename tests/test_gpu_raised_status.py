"""While the device status is raised (here by a bad compaction index) the tensor-core calls leave their outputs as
they are, those whose work is split and put together by a second kernel too: that kernel must not write what an earlier
call left in the workspace.  Once the status is cleared the same calls give what they gave before it."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def randn(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def make(hq, hkv, m, rows):
    """A context with a prefix of m tokens, and a function that raises its status."""
    bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16 + 1, torch.bfloat16, rows, 4)
    k = randn((1, m, hkv, 128), 1)
    pid, _, _ = bc.put_prefix(1, k, -k)
    short, _, _ = bc.reserve_prefix(2, 4)

    def raise_status():
        bc.compact_prefix(pid, short, torch.full((1, 1, 4), m, dtype=torch.int32, device="cuda"))
        assert bc.device_status() == binding.ERR_INVALID
    return bc, pid, raise_status


@pytest.mark.parametrize("m,rows,launches", [(40, 1600, 2), (300, 20, 1)])       # ranges of rows and their sums; one kernel
def test_accumulated_weights(m, rows, launches):
    hq, hkv = 14, 2
    bc, pid, raise_status = make(hq, hkv, m, rows)
    q = randn((rows, hq, 128), 2)
    lse = torch.full((rows, hq), 5.0, device="cuda")
    start = torch.rand((hkv, m), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))

    def call(scores, q):
        bc.prefix_weights(0, [pid], [0], [rows], q, lse, scores, [0], scores_in=scores, decay=0.5)
        return scores
    before = bc.launch_count()
    want = call(start.clone(), q)
    assert bc.launch_count() == before + launches
    call(start.clone(), q * 2)                                    # the workspace holds another call's sums
    raise_status()
    scores = start.clone()
    call(scores, q)
    assert bc.device_status() == binding.ERR_INVALID
    assert torch.equal(scores, start)
    assert bc.device_status(clear=True) == binding.ERR_INVALID
    assert torch.equal(call(scores, q), want)


@pytest.mark.parametrize("kind,m,n,kernel,launches", [
    ("attend", 4000, 9, binding.KERNEL_KEY_RANGES, 2),            # few rows against a long prefix: ranges of the keys
    ("attend", 2000, 200, binding.KERNEL_TENSOR, 2),              # few row tiles: keys split
    ("attend_full", 16, 2000, binding.KERNEL_TENSOR, 2),
    ("attend", 20, 30, binding.KERNEL_TENSOR, 1)])                # one kernel
def test_attention(kind, m, n, kernel, launches):
    hq, hkv = 2, 1
    bc, pid, raise_status = make(hq, hkv, m, n)
    q, k, v = randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)

    def call(out, lse, q):
        if kind == "attend":
            bc.attend(0, [pid], [0], [n], q, k, v, out, lse)
        else:
            bc.attend_full(0, [0], [n], q, k, v, out, lse)
    want, want_lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
    before = bc.launch_count()
    call(want, want_lse, q)
    assert bc.launch_count() == before + launches and bc.last_attention_kernel() == kernel
    call(torch.zeros_like(q), None, -q)                           # the workspace holds another call's partial results
    raise_status()
    out, lse = torch.full_like(q, 3.0), torch.full((n, hq), 7.0, device="cuda")
    call(out, lse, q)
    assert bc.device_status() == binding.ERR_INVALID
    assert (out == 3.0).all() and (lse == 7.0).all()
    assert bc.device_status(clear=True) == binding.ERR_INVALID
    call(out, lse, q)
    assert bc.device_status() == binding.OK
    assert torch.equal(out, want) and torch.equal(lse, want_lse)

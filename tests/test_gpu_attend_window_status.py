"""Windowed attention and the device status: waits that run out (a budget of one SM cycle: every wait that is not already
complete gives up) are reported and leave a context that works again; while the status is raised the tensor-core forms
leave their outputs as they are, those whose keys are split among them."""
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
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


# heads, cached tokens, rows, kernel, launches: ranges of keys and their join; whole items; row tiles of 256
FORMS = [(14, 2, 20000, 5, binding.KERNEL_KEY_RANGES, 2), (32, 32, 700, 300, binding.KERNEL_KEY_RANGES, 1),
         (32, 32, 3500, 3500, binding.KERNEL_TENSOR, 1)]


class Case:
    def __init__(self, hq, hkv, m, n, kernel, launches):
        self.bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16 + 1, torch.bfloat16, n, 1)
        k = randn((1, m, hkv, 128), 1)
        self.pid = self.bc.put_prefix(1, k, k.flip(1))[0]
        self.short = self.bc.reserve_prefix(2, 4)[0]
        self.q = randn((n, hq, 128), 2)
        self.m, self.n = m, n
        before = self.bc.launch_count()
        self.want = self.call(self.q)
        assert self.bc.launch_count() == before + launches and self.bc.last_attention_kernel() == kernel
        assert self.bc.device_status() == binding.OK

    def call(self, q, fill=0.0):
        out, lse = torch.full_like(q, fill), torch.full(q.shape[:2], fill, device="cuda")
        self.bc.attend_window(0, [self.pid], [self.m], [self.m - self.n], [0], [self.n], q, out, lse, 4, self.m // 2, 0)
        return out, lse

    def check(self):
        out, lse = self.call(self.q)
        assert self.bc.device_status() == binding.OK
        assert torch.equal(out, self.want[0]) and torch.equal(lse, self.want[1])


@pytest.mark.parametrize("form", FORMS)
def test_waits_that_run_out(form):
    c = Case(*form)
    c.bc.set_wait_budget(1)
    c.call(c.q)
    assert c.bc.device_status() == binding.ERR_TIMEOUT        # sticky until cleared
    c.call(c.q)                                               # no work on a flagged context
    assert c.bc.device_status(clear=True) == binding.ERR_TIMEOUT
    assert c.bc.device_status() == binding.OK
    c.bc.set_wait_budget(0)
    c.check()


@pytest.mark.parametrize("form", FORMS)
def test_raised_status(form):
    c = Case(*form)
    c.call(-c.q)                                              # the workspace holds another call's partial results
    c.bc.compact_prefix(c.pid, c.short, torch.full((1, 1, 4), c.m, dtype=torch.int32, device="cuda"))
    assert c.bc.device_status() == binding.ERR_INVALID
    out, lse = c.call(c.q, 3.0)
    assert c.bc.device_status() == binding.ERR_INVALID
    assert (out == 3.0).all() and (lse == 3.0).all()
    assert c.bc.device_status(clear=True) == binding.ERR_INVALID
    c.check()


def test_tokens_are_moved_while_the_status_is_raised():
    c = Case(*FORMS[0])
    c.bc.compact_prefix(c.pid, c.short, torch.full((1, 1, 4), c.m, dtype=torch.int32, device="cuda"))
    k, v = randn((2, 2, 128), 5), randn((2, 2, 128), 6)
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    c.bc.append_tokens(0, [c.short], [1], [0], [2], k, v)
    c.bc.read_tokens(0, [c.short], [1], [0], [2], kb, vb)
    assert c.bc.device_status(clear=True) == binding.ERR_INVALID
    assert torch.equal(kb, k) and torch.equal(vb, v)

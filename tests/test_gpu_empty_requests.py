"""A request without rows says nothing about the tensors: where its row offset points must not change what the calls on
the tensor cores read of the queries, which kernel they choose, or what they answer."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding

pytestmark = pytest.mark.gpu
FAR = [0, 10 ** 6, 2 ** 31 + 5, 2 ** 40]                       # row offsets of the empty request


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def randn(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("hq,hkv,n,kernel", [(32, 32, 3601, binding.KERNEL_TENSOR), (32, 8, 3601, binding.KERNEL_TENSOR),
                                             (14, 2, 77, binding.KERNEL_KEY_RANGES)])
def test_windowed_attention(hq, hkv, n, kernel):
    """The last row tile of the request is not full, and its rows are the last of the tensor."""
    m = 3700
    bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, 3)
    k, v, q = randn((1, m, hkv, 128), 1), randn((1, m, hkv, 128), 2), randn((n, hq, 128), 3)
    pid = bc.put_prefix(1, k, v)[0]

    def call(*args):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        bc.attend_window(0, *args, q, out, lse, 4, 500, 0)
        assert bc.device_status() == binding.OK and bc.last_attention_kernel() == kernel
        return out, lse
    want = call([pid], [m], [m - n], [0], [n])
    for far in FAR:
        for got in (call([pid, pid], [m, m], [m - n, 0], [0, far], [n, 0]), call([-1, pid, pid], [0, m, 5], [9, m - n, 0], [far, 0, far], [0, n, 0])):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("path", [binding.PATH_TENSOR, binding.PATH_TENSOR_PAIRS])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2)])
def test_attention(hq, hkv, path):
    m, n = 300, 517
    bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, 3)
    bc.set_path(path)
    pk, q, k, v = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)
    pid = bc.put_prefix(1, pk, -pk)[0]

    def call(full, *args):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        (bc.attend_full if full else bc.attend)(0, *args, q, k, v, out, lse)
        assert bc.device_status() == binding.OK
        return out, lse
    for full in (False, True):
        ids = [] if full else [[pid]]
        want = call(full, *ids, [0], [n])
        for far in FAR:
            ids = [] if full else [[-1, pid, pid]]
            got = call(full, *ids, [far, 0, far], [0, n, 0])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

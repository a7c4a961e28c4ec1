"""GPU parity of the rotary calls where a call is more than one round of work: several rows to a block with a partial
last block, blocks and threads that take more than one row.

Tolerances as derived in test_gpu_rope.py (E for a cosine or sine, four fp32 roundings, one to the type)."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
E = 1.5e-7


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


@pytest.fixture(scope="module")
def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def make(hq, hkv, d, dtype):
    return binding.BiCache(1, hq, hkv, d, 8, dtype, 16, 1)


def rows_of(n, heads, d, dtype, seed, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((n, heads + pad, d), generator=g, device="cuda").to(dtype)[:, :heads]


def cos_sin(positions, freq):
    """[rows, pairs, 2] in fp64.  The frequency in turns is cut to 52 fraction bits; its product with the position,
    modulo a turn, is exact in 64-bit integers, and what the cut leaves over is added as a small angle."""
    p = np.asarray(positions, dtype=np.int64)[:, None]
    turns = np.asarray(freq, dtype=np.float64) / (2 * np.pi)
    cut = np.floor(turns * 2.0 ** 52 + 0.5)
    whole = (p.astype(np.uint64) * cut.astype(np.int64).astype(np.uint64)) & np.uint64((1 << 52) - 1)
    a = 2 * np.pi * (whole.astype(np.float64) / 2.0 ** 52 + p * (turns - cut / 2.0 ** 52))
    return np.stack([np.cos(a), np.sin(a)], axis=-1)


def check(got, x, table, interleaved, scale, dtype):
    """got against x [rows, heads, D] turned by table, times scale."""
    x64, got64 = workloads.to_f64(x), workloads.to_f64(got)
    pairs = table.shape[1]
    d = np.arange(pairs)
    i, j = (2 * d, 2 * d + 1) if interleaved else (d, d + pairs)
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    a, b = x64[..., i], x64[..., j]
    inner = abs(scale) * (np.abs(a) + np.abs(b)) * (E + 4 * 2.0 ** -24)
    for at, ref in ((i, scale * (a * c - b * s)), (j, scale * (b * c + a * s))):
        err = np.abs(got64[..., at] - ref)
        assert (err <= inner + (np.abs(ref) + inner) * torch.finfo(dtype).eps / 2).all(), err.max()
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,rot", [(3, 1, 128, 128), (6, 2, 64, 32), (2, 2, 96, 20)])   # all, part, not whole chunks
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rounds,more", [(8, 3), (17, 1)])        # rows: from 8 an SM on four to a block; past 16 in turns
def test_many_rows(sms, dtype, hq, hkv, d, rot, interleaved, rounds, more):
    rows = rounds * sms + more
    assert rows % 4 != 0
    bc = make(hq, hkv, d, dtype)
    q, k = rows_of(rows + 2, hq, d, dtype, 1, 1), rows_of(rows + 2, hkv, d, dtype, 2)
    freq = binding.rope_frequencies(rot, 10000.0)
    pos = torch.randint(-100, 1 << 20, (rows,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda",
                        dtype=torch.int32)
    turn = cos_sin(pos.cpu().numpy(), freq)
    qo, ko = torch.full_like(q, 3), torch.full_like(k, 3)
    bc.rope(freq, q[:rows], qo[:rows], k[:rows], ko[:rows], positions=pos, interleaved=interleaved, attention_scale=1.25)
    assert (qo[rows:] == 3).all() and (ko[rows:] == 3).all()      # rows behind the last
    check(qo[:rows], q[:rows], turn, interleaved, 1.25, dtype)
    check(ko[:rows], k[:rows], turn, interleaved, 1.25, dtype)
    q2, k2 = q.clone(), k.clone()                                 # in place
    bc.rope(freq, q2[:rows], q2[:rows], k2[:rows], k2[:rows], positions=pos, interleaved=interleaved, attention_scale=1.25)
    assert torch.equal(q2[:rows], qo[:rows]) and torch.equal(k2[:rows], ko[:rows])
    assert torch.equal(q2[rows:], q[rows:]) and torch.equal(k2[rows:], k[rows:])
    back = torch.empty_like(k)
    bc.rope(freq, None, None, ko[:rows], back[:rows], positions=pos, interleaved=interleaved, attention_scale=1.25, inverse=True)
    check(back[:rows], ko[:rows], turn * np.array([1.0, -1.0]), interleaved, 1 / 1.25, dtype)


@pytest.mark.parametrize("rot,rows", [(128, 5003), (256, 2501), (96, 3001), (20, 20001), (2, 310001)])
def test_table_of_more_rows_than_threads(sms, rot, rows):
    per_thread = rows / (2 * sms * (256 // (rot // 2)))
    assert per_thread > 1                                         # every thread takes more than one row, most several
    bc = make(2, 1, 128, torch.bfloat16)
    freq = binding.rope_frequencies(rot, 10000.0)
    table = torch.full((rows + 1, rot // 2, 2), 9.0, device="cuda")
    pos = torch.randint(-5, 1 << 20, (rows,), generator=torch.Generator(device="cuda").manual_seed(rot), device="cuda",
                        dtype=torch.int32)
    for positions, at in ((pos, pos.cpu().numpy()), (None, np.arange(777, 777 + rows))):
        bc.rope_table(freq, table[:rows], positions=positions, position0=777, attention_scale=1.5)
        err = np.abs(workloads.to_f64(table[:rows]) - 1.5 * cos_sin(at, freq))
        assert (err <= 1.5 * (E + 2 * 2.0 ** -24)).all(), err.max()
        assert (table[rows] == 9.0).all()

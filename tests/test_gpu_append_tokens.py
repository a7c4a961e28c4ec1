"""GPU parity of appending tokens to stored prefixes and reading them back, against the fp64 oracle and bit for bit.

Values and unrotated keys are bit-exact.  Rotated keys and queries: the tolerance of the rotary calls (cosine and sine off by
E = 1.5e-7, four fp32 roundings of at most (|a| + |b|) scale, one rounding to the type of half a step)."""
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


def randn(shape, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def garbage(bc):
    """All bits set: every number in the pools is a NaN."""
    bc.k_pool.fill_(255)
    bc.v_pool.fill_(255)


def check_rotated(got, x, positions, freq, axis, interleaved, scale, dtype):
    ref = gc.rope_axes(f64(x), positions, freq, axis, interleaved, scale)
    pairs, ax = len(freq), np.abs(f64(x))
    size = np.zeros_like(ax)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        size[..., a] = size[..., b] = ax[..., a] + ax[..., b]
    inner = abs(scale) * size * (E + 4 * 2.0 ** -24)
    err = np.abs(f64(got) - ref)
    assert (err <= inner + (np.abs(ref) + inner) * torch.finfo(dtype).eps / 2).all(), err.max()
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# prefix lengths, tokens, rows: page ends, last pages, one token, whole prefixes, an empty request, one prefix twice
BATCH = dict(m=[40, 16, 17, 100, 33, 5], pid=[0, 1, 2, 3, 4, 0, 5, 3], tok=[0, 15, 0, 30, 32, 30, 2, 99],
             n=[30, 1, 17, 50, 1, 10, 0, 1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,rot,axes", [(7, 1, 128, 128, 1), (4, 4, 64, 64, 3), (2, 1, 128, 32, 2), (3, 3, 96, 20, 1),
                                               (6, 2, 128, 2, 1), (2, 2, 256, 256, 4), (28, 4, 128, 108, 3), (1, 1, 32, 30, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_batch(dtype, hq, hkv, d, rot, axes, interleaved):
    bc = binding.BiCache(2, hq, hkv, d, 20, dtype, 16, 1, free_order=np.random.default_rng(3).permutation(20))
    garbage(bc)
    ids = [bc.reserve_prefix(i + 1, m)[0] for i, m in enumerate(BATCH["m"])]
    pid = [ids[i] for i in BATCH["pid"]]
    off, rows = [], 3                                          # rows behind, before and between the requests'
    for n in BATCH["n"]:
        off.append(rows)
        rows += n + (n == 17)
    rows += 2
    packed = randn((rows, hq + 2 * hkv + 1, d), 1, dtype)      # rows of one tensor, as a fused projection writes them
    q, k, v = packed[:, :hq], packed[:, hq:hq + hkv], packed[:, hq + hkv:hq + 2 * hkv]
    q_out = torch.full((rows, hq, d), 7.0, dtype=dtype, device="cuda")
    freq = binding.rope_frequencies(rot, 10000.0)
    axis = [i % axes for i in range(rot // 2)]
    pos = torch.randint(-5, 1 << 20, (axes, rows + 3), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()[:, :rows]
    r = binding.Rotation(freq, interleaved, 1.25, axis, axes)
    bc.append_tokens(1, pid, BATCH["tok"], off, BATCH["n"], k, v, q, q_out, r, pos)
    k_back, v_back = torch.full_like(k.contiguous(), 5.0), torch.full_like(v.contiguous(), 5.0)
    bc.read_tokens(1, pid, BATCH["tok"], off, BATCH["n"], k_back, v_back)
    assert bc.device_status() == 0
    mine = torch.zeros(rows, dtype=torch.bool)
    for o, n in zip(off, BATCH["n"]):
        mine[o:o + n] = True
    mine = mine.cuda()
    assert same(v_back[mine], v[mine])
    p = [pos[a][mine].tolist() for a in range(axes)]
    check_rotated(k_back[mine], k[mine], p, freq, axis, interleaved, 1.25, dtype)
    check_rotated(q_out[mine], q[mine], p, freq, axis, interleaved, 1.25, dtype)
    assert (q_out[~mine] == 7).all() and (k_back[~mine] == 5).all() and (v_back[~mine] == 5).all()
    # the tokens that were not written, and the other layer, hold what they held; the slots behind the end of the
    # prefixes whose last page was written are zero
    full = binding.BiCache(1, hq, hkv, d, 20, dtype, 16, 1)
    for i, m in enumerate(BATCH["m"]):
        written = torch.zeros(m, dtype=torch.bool)
        for j, t, n in zip(BATCH["pid"], BATCH["tok"], BATCH["n"]):
            if j == i:
                written[t:t + n] = True
        a, b = torch.empty((m, hkv, d), dtype=dtype, device="cuda"), torch.empty((m, hkv, d), dtype=dtype, device="cuda")
        bc.read_prefix_layer(ids[i], 1, a, b)
        for x in (a, b):
            assert x[(~written).cuda()].isnan().all() and not x[written.cuda()].isnan().any()
        bc.read_prefix_layer(ids[i], 0, a, b)
        assert a.isnan().all() and b.isnan().all()
        es, page = a.element_size(), bc.prefix_pages(ids[i], 1)[-1]
        for pool in (bc.k_pool, bc.v_pool):
            last = pool.view(2, 20, -1)[1, page].clone()
            values = last.view(dtype).view(hkv, -1)
            zeros = (values == 0).sum(1)
            want = (16 - m % 16) % 16 * d if written[(m - 1) // 16 * 16:].any() else 0
            assert (zeros == want).all(), (i, zeros, want)
    # queries in place: the same bits
    q2 = q.contiguous()
    bc.append_tokens(1, pid, BATCH["tok"], off, BATCH["n"], k, v, q2, q2, r, pos)
    q_out[~mine] = q[~mine]
    assert same(q2, q_out)


@pytest.mark.parametrize("dtype,hq,hkv,d", [(torch.bfloat16, 4, 2, 128), (torch.float32, 3, 1, 64)])
def test_positions_are_token_indices_and_plain_copies(dtype, hq, hkv, d):
    bc = binding.BiCache(1, hq, hkv, d, 20, dtype, 16, 1)
    garbage(bc)
    ids = [bc.reserve_prefix(i, m)[0] for i, m in ((1, 100), (2, 31))]
    k, v, q = randn((31, hkv, d), 1, dtype), randn((31, hkv, d), 2, dtype), randn((31, hq, d), 3, dtype)
    freq = binding.rope_frequencies(d, 10000.0)
    q_out, kb, vb = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    args = (0, ids, [77, 9], [0, 11], [11, 20])
    where = [list(range(77, 88)) + list(range(9, 29))]
    bc.append_tokens(*args, k, v, q, q_out, binding.Rotation(freq))
    bc.read_tokens(*args, kb, vb)
    check_rotated(kb, k, where, freq, [0] * (d // 2), False, 1.0, dtype)
    check_rotated(q_out, q, where, freq, [0] * (d // 2), False, 1.0, dtype)
    assert same(vb, v)
    bc.append_tokens(*args, k, v)                              # no rotation
    bc.read_tokens(*args, kb, vb)
    assert same(kb, k) and same(vb, v)
    k_nan = k.clone()
    k_nan[3, 0, 5], k_nan[4, 0, 6] = float("nan"), float("inf")
    bc.append_tokens(*args, k_nan, v)
    bc.read_tokens(*args, kb, vb)
    assert same(kb, k_nan)


def test_a_whole_prefix_written_this_way_is_the_prefix_that_is_put():
    hq, hkv, d, m = 14, 2, 128, 1500
    k, v = randn((1, m, hkv, d), 1, torch.bfloat16), randn((1, m, hkv, d), 2, torch.bfloat16)
    q, own = randn((20, hq, d), 3, torch.bfloat16), randn((20, hkv, d), 4, torch.bfloat16)
    outs = []
    for way in range(2):
        bc = binding.BiCache(1, hq, hkv, d, 100, torch.bfloat16, 64, 2)
        garbage(bc)
        if way == 0:
            pid = bc.put_prefix(1, k, v)[0]
        else:
            pid = bc.reserve_prefix(1, m)[0]
            cuts = [0, 1, 5, 700, 1489, 1500]
            bc.append_tokens(0, [pid] * 5, cuts[:-1], cuts[:-1], np.diff(cuts), k[0], v[0])
        out = torch.empty_like(q)
        bc.attend(0, [pid], [0], [20], q, own, own, out)
        assert bc.device_status() == 0
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and outs[0].isfinite().all()


@pytest.mark.parametrize("tokens", [1, 31, 32 * 148 - 1, 32 * 148 + 3, 20000])      # one row to a block, four rows
def test_many_rows(tokens):
    hq, hkv, d = 2, 1, 128
    bc = binding.BiCache(1, hq, hkv, d, 1300, torch.bfloat16, 16, 1)
    pid = bc.reserve_prefix(1, tokens)[0]
    k, v, q = randn((tokens, hkv, d), 1, torch.bfloat16), randn((tokens, hkv, d), 2, torch.bfloat16), randn((tokens, hq, d), 3, torch.bfloat16)
    r = binding.Rotation(binding.rope_frequencies(d, 10000.0))
    q_out, kb, vb = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    bc.append_tokens(0, [pid], [0], [0], [tokens], k, v, q, q_out, r)
    bc.read_tokens(0, [pid], [0], [0], [tokens], kb, vb)
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    bc.rope(binding.rope_frequencies(d, 10000.0), q, want_q, k, want_k)
    assert same(kb, want_k) and same(q_out, want_q) and same(vb, v)


@pytest.mark.parametrize("seed", range(16))
def test_random_runs(seed):
    """Disjoint runs of tokens of several prefixes in any order, against what the rotary call makes of the same rows."""
    rng = np.random.default_rng(seed)
    hq, hkv, d = [(7, 1, 128), (4, 4, 64), (2, 2, 96), (32, 8, 128)][seed % 4]
    dtype = torch.float32 if seed % 3 == 0 else torch.bfloat16
    lens = [int(x) for x in np.exp(rng.uniform(0, 7, rng.integers(1, 7)))]
    pages = sum((m + 15) // 16 for m in lens)
    bc = binding.BiCache(2, hq, hkv, d, pages, dtype, 16, 1, free_order=rng.permutation(pages) if seed % 2 else None)
    garbage(bc)
    ids = [bc.reserve_prefix(i, m)[0] for i, m in enumerate(lens)]
    runs = []
    for i, m in enumerate(lens):
        cuts = sorted(set([0, m] + rng.integers(0, m + 1, 4).tolist()))
        runs += [(i, a, b - a) for a, b in zip(cuts, cuts[1:]) if rng.random() < 0.8]
    rng.shuffle(runs)
    runs = [tuple(int(x) for x in r) for r in runs] or [(0, 0, lens[0])]
    pid, tok, n = [ids[i] for i, _, _ in runs], [t for _, t, _ in runs], [k for _, _, k in runs]
    off = (np.concatenate([[0], np.cumsum(n)[:-1]]) + np.arange(len(n))).tolist()          # a row between two runs
    rows = off[-1] + n[-1]
    q, k, v = (randn((rows, h, d), seed * 3 + j, dtype) for j, h in enumerate((hq, hkv, hkv)))
    where = torch.zeros(rows, dtype=torch.int32)
    for o, t, c in zip(off, tok, n):
        where[o:o + c] = torch.arange(t, t + c)
    rot = int(rng.choice([d, d // 2, 2 * rng.integers(1, d // 2 + 1)]))
    inter, freq = bool(rng.integers(0, 2)), binding.rope_frequencies(rot, 10000.0)
    q_out, kb, vb = torch.full_like(q, 3.0), torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    bc.append_tokens(1, pid, tok, off, n, k, v, q, q_out, binding.Rotation(freq, inter))
    bc.read_tokens(1, pid, tok, off, n, kb, vb)
    mine = torch.zeros(rows, dtype=torch.bool)
    for o, c in zip(off, n):
        mine[o:o + c] = True
    mine = mine.cuda()
    axis, p = [0] * (rot // 2), [where[mine.cpu()].tolist()]
    check_rotated(q_out[mine], q[mine], p, freq, axis, inter, 1.0, dtype)
    check_rotated(kb[mine], k[mine], p, freq, axis, inter, 1.0, dtype)
    assert same(vb[mine], v[mine])
    for x in (q_out, kb, vb):
        assert (x[~mine] == 3).all()
    for i, m in enumerate(lens):                               # by the call that reads whole layers
        a, b = torch.empty((m, hkv, d), dtype=dtype, device="cuda"), torch.empty((m, hkv, d), dtype=dtype, device="cuda")
        bc.read_prefix_layer(ids[i], 1, a, b)
        rest = torch.ones(m, dtype=torch.bool)
        for (j, t, c), o in zip(runs, off):
            if j == i:
                assert same(a[t:t + c], kb[o:o + c]) and same(b[t:t + c], vb[o:o + c])
                rest[t:t + c] = False
        assert a[rest.cuda()].isnan().all() and b[rest.cuda()].isnan().all()


def test_lists_that_take_several_launches():
    hkv, d = 1, 32
    # 600 short requests of 8 words and a page each, and one whose pages alone are too many
    lengths = [1 + i % 20 for i in range(600)] + [130000]
    pages = sum((n + 15) // 16 for n in lengths)
    bc = binding.BiCache(1, 1, hkv, d, pages, torch.bfloat16, 16, 1, free_order=np.random.default_rng(0).permutation(pages))
    garbage(bc)
    ids = [bc.reserve_prefix(i, n)[0] for i, n in enumerate(lengths)]
    off = np.concatenate([[0], np.cumsum(lengths)[:-1]])
    k, v = randn((sum(lengths), hkv, d), 1, torch.bfloat16), randn((sum(lengths), hkv, d), 2, torch.bfloat16)
    before = bc.launch_count()
    bc.append_tokens(0, ids, [0] * 601, off, lengths, k, v)
    assert 2 <= bc.launch_count() - before <= 4
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    bc.read_tokens(0, ids, [0] * 601, off, lengths, kb, vb)
    assert same(kb, k) and same(vb, v)
    a, b = torch.empty((130000, hkv, d), dtype=k.dtype, device="cuda"), torch.empty((130000, hkv, d), dtype=k.dtype, device="cuda")
    bc.read_prefix_layer(ids[600], 0, a, b)
    assert same(a, k[off[600]:]) and same(b, v[off[600]:])

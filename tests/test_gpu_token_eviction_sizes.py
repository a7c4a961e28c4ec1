"""GPU parity of the token-eviction calls where a call is more than one round of work: items of many row tiles, more
prefixes than a launch takes, more rows of scores than the GPU works on at a time, blocks that copy more than one round
of rows, page lists that do not fit the launch parameters.

Tolerance of a weight exp(scale q.k - lse), relative, from the inputs (x: the exponent in units of log 2):
  products   D additions in fp32, each rounded or cut: D 2^-23 sum |q_d k_d| |scale|
  scale      times log2(e) as fp32, two roundings of 2^-24 and the constant's: 2^-22 |scale| sum |q_d k_d| covers them
  lse        times log2(e) in fp32, and the rounding of x: 2^-22 |lse| and the term above cover them
  exp        2 units in the last place: 2^-22
  sums       positive terms, so an addition costs half a step of its result: 48 tiles on a lane, 5 steps across the
             lanes, 1 for the sum carried over such runs of tiles (its own error is carried along), 3 across the lane groups,
             1 for a range's partial sum; ranges in fp64.  On the CUDA cores 8 in fp32, 1 for a partial sum, the rest in fp64
  result     one rounding for each launch that adds to it; in all not above 66 roundings of 2^-24 for up to 8 launches"""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
SCALE = float(np.float32(0.11))                                   # exact in the call's float


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


@pytest.fixture(scope="module")
def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, seed, dtype, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def check_weights(got, k, q, lse, before=None, decay=0.0):
    """got [Hkv, m] against the definition in 64 bits, one query head at a time."""
    m, hkv, d = k.shape
    group = q.shape[1] // hkv
    want = torch.zeros((hkv, m), dtype=torch.float64, device="cuda") if before is None else decay * before.double()
    size = 0.0
    for h in range(q.shape[1]):
        live = ~torch.isinf(lse[:, h])
        k64, q64, l64 = k[:, h // group].double(), q[live, h].double(), lse[live, h].double()
        if len(l64):
            want[h // group] += torch.exp(SCALE * (k64 @ q64.T) - l64).sum(1)
            size = max(size, float((k64.abs() @ q64.abs().T).max()))
    finite = lse[torch.isfinite(lse)]
    far = float(finite.abs().max()) if len(finite) else 0.0
    rel = SCALE * size * (d * 2.0 ** -23 + 2.0 ** -22) + far * 2.0 ** -22 + 2.0 ** -22 + 66 * 2.0 ** -24
    err = (got.double() - want).abs()
    assert (err <= rel * want.abs() + 2.0 ** -126).all(), ((err / want.abs()).max(), rel)


@pytest.mark.parametrize("heads,tokens", [((16, 1, 128), [800]), ((14, 1, 128), [511, 1, 0, 380]), ((6, 2, 128), [2500, 1611])])
def test_items_of_more_row_tiles_than_a_thread_adds_at_once(sms, heads, tokens):
    """As many blocks of keys as SMs, so the rows are not split: an item has some hundred row tiles, which a thread adds in
    runs of 48 and a rest.  One launch shows that they are not split."""
    hq, hkv, d = heads
    rows, m = sum(tokens), 256 * (sms // hkv) - 5
    assert rows // (128 // (hq // hkv)) > 96                      # more than two runs of tiles
    bc = binding.BiCache(1, hq, hkv, d, (m + 15) // 16, torch.bfloat16, 16, 4)
    k, q = randn((m, hkv, d), 1, torch.bfloat16), randn((rows, hq, d), 2, torch.bfloat16, 1.5)
    pid, _, _ = bc.put_prefix(1, k[None], k[None])
    off = np.cumsum([0] + tokens[:-1]).tolist()
    for dead in (False, True):
        lse = torch.rand((rows, hq), generator=gen(3), device="cuda") * 4 + 3
        if dead:                                                  # rows, whole tiles and whole runs that add nothing
            lse[torch.rand((rows,), generator=gen(4), device="cuda") < 0.1] = INF
            lse[rows // 2:rows // 2 + 300] = -INF
            q[rows // 2 + 7] = NAN
        start = torch.rand((hkv, m), generator=gen(5), device="cuda")
        out = start.clone()
        launches = bc.launch_count()
        bc.prefix_weights(0, [pid] * len(tokens), off, tokens, q, lse, out, [0] * len(tokens), scores_in=out, decay=0.5,
                          scale=SCALE)
        assert bc.launch_count() == launches + 1
        check_weights(out, k, q, lse, start, 0.5)
    assert bc.device_status() == 0


@pytest.mark.parametrize("dtype,d,groups", [(torch.bfloat16, 128, 70), (torch.bfloat16, 128, 450), (torch.float32, 64, 450)])
def test_a_prefix_for_every_request(dtype, d, groups):
    hq, hkv = 4, 2
    lengths = [1 + (37 * i) % 61 for i in range(groups)]
    counts = [(5 * i) % 4 for i in range(groups)]                 # a quarter of the requests are empty
    bc = binding.BiCache(1, hq, hkv, d, sum((m + 15) // 16 for m in lengths), dtype, 16, groups)
    q = randn((sum(counts), hq, d), 2, dtype, 1.5)
    lse = torch.rand((sum(counts), hq), generator=gen(3), device="cuda") * 4 + 3
    ks = [randn((m, hkv, d), 100 + i, dtype) for i, m in enumerate(lengths)]
    ids = [bc.put_prefix(i + 1, k[None], k[None])[0] for i, k in enumerate(ks)]
    off = np.cumsum([0] + counts[:-1])
    start = torch.rand((groups, hkv, 64), generator=gen(5), device="cuda")
    out = torch.full_like(start, 9.0)
    bc.prefix_weights(0, ids, off, counts, q, lse, out, [i * hkv * 64 for i in range(groups)], scores_in=start, decay=0.5,
                      scale=SCALE)
    for i, (m, n, at) in enumerate(zip(lengths, counts, off)):
        check_weights(out[i, :, :m], ks[i], q[at:at + n], lse[at:at + n], start[i, :, :m], 0.5)
        assert (out[i, :, m:] == 9.0).all()
    assert bc.device_status() == 0


# ---------------------------------------------------------------------------------------------
# choice of tokens
# ---------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def bc():
    return binding.BiCache(1, 2, 1, 128, 8, torch.bfloat16, 16, 1)


def check_select(bc, scores, keep, first=0, last=0):
    rows, n = scores.shape
    idx = torch.full((rows, keep + 1), -7, dtype=torch.int32, device="cuda")
    bc.select_tokens(scores, keep, idx[:, :keep], first, last)
    first = min(first, n)
    protected = torch.zeros(n, dtype=torch.bool, device="cuda")
    protected[:first] = True
    protected[n - min(last, n - first):] = True
    s = torch.where(torch.isnan(scores), -INF, scores.double()) + 0.0            # -0 equals +0
    order = torch.sort(s, dim=1, descending=True, stable=True).indices           # equal scores by index
    order = order.gather(1, torch.sort(protected[order], dim=1, descending=True, stable=True).indices)
    assert torch.equal(idx[:, :keep].long(), order[:, :keep].sort(dim=1).values), (keep, first, last)
    assert (idx[:, keep] == -7).all()


def scores_of(rows, n, seed, pad=1):
    """Weights as they are (positive, heavy-tailed, some rows of many equal ones), rows that start off alignment."""
    x = torch.exp(torch.randn((rows, n + pad), generator=gen(seed), device="cuda") * 2 - 5)
    x[1::3] = (x[1::3] * 64).round()
    x[2::3, n // 2:] = 0
    return x[:, pad:]


@pytest.mark.parametrize("n", [1, 3, 33, 1000, 5001, 40001])
def test_more_rows_than_sms(bc, sms, n):
    x = scores_of(2 * sms + 5, n, n)
    for keep, first, last in ((1, 0, 0), ((n + 1) // 2, min(2, (n + 1) // 2), 0), (n, 1, 1)):
        check_select(bc, x, keep, first, last)


@pytest.mark.parametrize("n,blocks", [(60001, 2), (150001, 4), (300007, 8)])
def test_more_rows_than_clusters(bc, sms, n, blocks):
    rows = sms // blocks + 7                                      # clusters of `blocks` blocks, a block to an SM
    check_select(bc, scores_of(rows, n, n), n // 4, 4, 33)


def test_rows_that_are_read_in_every_pass(bc):
    """Rows too long to stay on chip: every start relative to 16 bytes, values of every kind, rows of one value."""
    n = 393301
    vals = torch.tensor([NAN, INF, -INF, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0, -1.0, -NAN], device="cuda")
    x = torch.randn((4, n + 2), generator=gen(1), device="cuda")  # a row is 3 scores past a multiple of 4 longer than the last
    x[1] = vals[torch.randint(0, len(vals), (n + 2,), generator=gen(2), device="cuda")]
    x[3] = (x[3] * 3).round()
    for pad in (0, 1, 2):                                         # rows start 0 .. 3 scores past a 16-byte boundary
        for keep, first, last in ((1, 0, 0), (n // 3, 4, 64), (n - 5, 0, 1), (n, 3, 2), (70, 30, 40)):
            check_select(bc, x[:, pad:pad + n], keep, first, last)
    for v in vals.tolist():
        check_select(bc, torch.full((1, n), v, device="cuda"), 1000, 3, 5)


# ---------------------------------------------------------------------------------------------
# copies
# ---------------------------------------------------------------------------------------------

def read(bc, pid, layer, m, pad=0):
    """A layer of a prefix, into strided rows, with rows behind the last that have to stay."""
    wide = torch.full((2, m + 1, bc.Hkv + pad, bc.D), 5.0, dtype=bc.dtype, device="cuda")
    k, v = wide[0][:, :bc.Hkv], wide[1][:, :bc.Hkv]
    bc.read_prefix_layer(pid, layer, k[:m], v[:m])
    assert (wide[:, m] == 5.0).all() and (wide[:, :, bc.Hkv:] == 5.0).all()
    return k[:m], v[:m]


def test_more_rows_than_one_round_of_blocks_copies(sms):
    hkv, d, layers = 8, 128, 2
    m, keep = 64 * sms * 16 // hkv + 1003, 64 * sms * 16 // hkv + 101     # 16 rows (of a token and head) to a block
    pages = (m + 15) // 16 + (keep + 15) // 16
    bc = binding.BiCache(layers, hkv, hkv, d, pages, torch.bfloat16, 16, 1, free_order=workloads.shuffled_page_order(pages, 3))
    k, v = randn((layers, m, hkv, d), 1, torch.bfloat16), randn((layers, m, hkv, d), 2, torch.bfloat16)
    src, _, _ = bc.put_prefix(1, k, v)
    dst, _, _ = bc.reserve_prefix(2, keep)
    idx = torch.randint(0, m, (layers, hkv, keep), generator=gen(4), device="cuda", dtype=torch.int32)
    bc.compact_prefix(src, dst, idx)
    for l in range(layers):
        gk, gv = read(bc, src, l, m, 1)
        assert torch.equal(gk, k[l]) and torch.equal(gv, v[l])
        gk, gv = read(bc, dst, l, keep, 1)
        for h in range(hkv):
            assert torch.equal(gk[:, h], k[l, idx[l, h].long(), h]) and torch.equal(gv[:, h], v[l, idx[l, h].long(), h])
    assert bc.device_status() == 0


@pytest.mark.parametrize("pages", [7936, 7937, 9001])
def test_read_back_of_more_pages_than_the_launch_parameters_hold(pages):
    m = 16 * pages - 3
    bc = binding.BiCache(2, 1, 1, 32, pages, torch.float32, 16, 1, free_order=workloads.shuffled_page_order(pages, 1))
    k = randn((2, m, 1, 32), 1, torch.float32)
    pid, _, _ = bc.put_prefix(1, k, -k)
    for l in (1, 0):
        gk, gv = read(bc, pid, l, m, 1)
        assert torch.equal(gk, k[l]) and torch.equal(gv, -k[l])

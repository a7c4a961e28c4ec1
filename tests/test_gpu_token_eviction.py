"""GPU parity of token eviction (prefix_weights, select_tokens, compact_prefix) against the fp64 oracle.

Tolerance of the weights, derived per call from the inputs.  A weight is 2^x, x = s l2e scale - lse l2e with
s = q.k; relative error of the weight = ln 2 * (absolute error of x) + the exponential's.
  s:       D products, each sum rounded (or cut) to fp32: D 2^-23 sum |q_d k_d|, times |scale| on the way to the exponent
  scale:   scale * log2(e) as fp32, two roundings of 2^-24 and the constant's: 1.5 * 2^-23 |scale s|
  lse:     times log2(e) in fp32: 2^-23 |lse|
  x:       one rounding: 2^-24 (|scale s| + |lse|)
  exp:     2 units in the last place (2^-22); the CUDA-core path's expf the same
  sums:    64 additions per row tile in fp32, all of one sign (64 * 2^-24), the rest compensated or fp64
  result:  rounded to fp32: 2^-24, once per launch
The sum of positive terms has the terms' largest relative error."""
import numpy as np
import pytest
import torch

import oracle
import __graft_entry__ as entry
from oracle import token_ops as op
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
SCALE = float(np.float32(0.11))                                   # exact in the call's float


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def f64(t):
    return workloads.to_f64(t)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, seed, dtype, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


class Batch:
    """Prefixes of given lengths, requests per prefix, queries and plausible log-sum-exps."""

    def __init__(self, heads, dtype, prefixes, suffixes, seed=5, layers=1, q_pad=0, path=binding.PATH_AUTO, extra=0):
        self.hq, self.hkv, self.d = heads
        self.g = self.hq // self.hkv
        pages = sum((m + 15) // 16 for m in prefixes) + extra
        order = workloads.shuffled_page_order(pages, seed)
        self.rows = sum(sum(n) for n in suffixes) + 3              # rows behind the last request
        self.bc = binding.BiCache(layers, self.hq, self.hkv, self.d, pages, dtype, max(self.rows, 16), 64, free_order=order)
        self.bc.set_path(path)
        self.m = list(prefixes)
        self.k, self.pid = [], []
        for i, m in enumerate(prefixes):
            k = randn((layers, m, self.hkv, self.d), seed * 100 + i, dtype)
            pid, _, _ = self.bc.put_prefix(i + 1, k, -k)
            self.k.append(k)
            self.pid.append(pid)
        wide = randn((self.rows, self.hq + q_pad, self.d), seed * 100 + 77, dtype, 1.5)
        self.q = wide[:, :self.hq]
        self.ids, self.off, self.n, self.slice = [], [], [], []
        row = 0
        for pid, ns in zip(self.pid, suffixes):
            self.slice.append((row, row + sum(ns)))
            for n in ns:
                self.ids.append(pid)
                self.off.append(row)
                self.n.append(n)
                row += n
        self.lse = torch.rand((self.rows, self.hq), generator=gen(seed + 1), device="cuda") * 4 + 3
        self.mmax = max(prefixes) + 5
        self.so = [i * self.hkv * self.mmax for i, ns in enumerate(suffixes) for _ in ns]

    def fresh(self, seed=9):
        return torch.rand((len(self.m), self.hkv, self.mmax), generator=gen(seed), device="cuda")

    def run(self, out, sin=None, decay=0.0, layer=0):
        self.bc.prefix_weights(layer, self.ids, self.off, self.n, self.q, self.lse, out, self.so, scores_in=sin,
                               decay=decay, scale=SCALE)
        return out

    def check(self, out, before=None, decay=0.0, layer=0, untouched=None):
        assert self.bc.device_status() == 0
        got = f64(out)
        for i, m in enumerate(self.m):
            a, b = self.slice[i]
            q, lse, k = f64(self.q)[a:b], f64(self.lse)[a:b], f64(self.k[i][layer])
            ref = op.prefix_weights(k, q, lse, self.g, SCALE, None if before is None else f64(before)[i], decay)
            s_abs = 0.0
            for h in range(self.hq):
                live = np.isfinite(lse[:, h])
                if live.any():
                    s_abs = max(s_abs, float((np.abs(k[:, h // self.g]) @ np.abs(q[live, h]).T).max()))
            l_max = np.abs(lse[np.isfinite(lse)]).max() if np.isfinite(lse).any() else 0.0
            rel = SCALE * s_abs * (self.d * 2.0 ** -23 + 2.0 ** -22) + l_max * 2.0 ** -22 + 2.0 ** -22 + 66 * 2.0 ** -24
            err = np.abs(got[i, :, :m] - ref)
            assert (err <= rel * np.abs(ref) + 2.0 ** -126).all(), (m, (err / np.abs(ref)).max(), rel)
            if untouched is not None:
                assert (got[i, :, m:] == f64(untouched)[i, :, m:]).all()       # columns behind the prefix


MHA, GQA7, GQA3, MQA = (4, 4, 128), (14, 2, 128), (6, 2, 128), (16, 1, 128)


@pytest.mark.parametrize("heads,prefixes,suffixes", [
    (MHA, [1], [[1]]), (GQA7, [16], [[1]]), (MQA, [17], [[3]]), (GQA3, [128], [[43]]), (MHA, [129], [[128]]),
    (GQA7, [255], [[1, 0, 36]]), (GQA3, [256], [[129, 1]]), (MQA, [257], [[5, 16, 2]]),
    (MHA, [100, 300, 15], [[7, 1], [130, 64], [200]]), (GQA7, [513, 40], [[9], [18, 19, 0, 21]]),
    (MHA, [64, 31], [[0, 0], [5]]), (MQA, [1023], [[300]]), ((130, 1, 128), [70], [[3]]), ((128, 1, 128), [40], [[2, 1]]),
    ((65, 1, 128), [300], [[2, 9]]), ((10, 2, 128), [260], [[100, 3, 77]]), ((48, 1, 128), [20], [[40]]),
])
@pytest.mark.parametrize("path", [binding.PATH_AUTO, binding.PATH_SIMT])
def test_weights(heads, prefixes, suffixes, path):
    b = Batch(heads, torch.bfloat16, prefixes, suffixes, path=path, q_pad=1)
    out = b.fresh()
    was = out.clone()
    b.check(b.run(out), untouched=was)
    sin = b.fresh(10)
    b.check(b.run(out, sin, 0.75), sin, 0.75, untouched=was)
    keep = sin.clone()
    b.run(sin, sin, 1.0)                                          # in place
    b.check(sin, keep, 1.0, untouched=keep)


@pytest.mark.parametrize("dtype,heads", [(torch.float32, (4, 4, 64)), (torch.float32, (6, 2, 128)), (torch.float32, (3, 1, 32)),
                                         (torch.float32, (2, 2, 256)), (torch.bfloat16, (8, 2, 64)), (torch.bfloat16, (5, 1, 96))])
def test_weights_other_types_and_head_dims(dtype, heads):
    b = Batch(heads, dtype, [65, 200, 1], [[33, 64], [1, 0, 5], [130]], q_pad=2)
    out, sin = b.fresh(), b.fresh(10)
    b.check(b.run(out, sin, 0.5), sin, 0.5)


@pytest.mark.parametrize("dtype,heads,prefixes,suffixes", [
    (torch.float32, (4, 4, 64), [1500, 77], [[700, 3], [129]]), (torch.float32, (4, 2, 192), [3001], [[150, 1]]),
    (torch.float32, (2, 2, 224), [3001], [[150, 1]]), (torch.bfloat16, (6, 2, 64), [4100], [[90, 17]]),
    (torch.bfloat16, (4, 4, 160), [2500], [[128]]), (torch.float32, (5, 1, 32), [129, 10000], [[16], [17]])])
def test_weights_that_fill_the_gpu(dtype, heads, prefixes, suffixes):
    """Batches with a block of keys for every SM, where a thread takes more keys if they fit."""
    b = Batch(heads, dtype, prefixes, suffixes, q_pad=1)
    out, sin = b.fresh(), b.fresh(10)
    b.check(b.run(out, sin, 0.5), sin, 0.5)


@pytest.mark.parametrize("dtype,heads", [(torch.bfloat16, GQA7), (torch.float32, (4, 2, 64))])
def test_rows_without_a_log_sum_exp_add_nothing(dtype, heads):
    b = Batch(heads, dtype, [300, 20], [[70, 33], [12]])
    b.lse[3] = INF
    b.lse[40:75] = -INF
    b.lse[80, 1] = INF
    b.lse[103:] = INF                                             # every row of the second prefix
    b.q[3] = NAN                                                  # what such a row holds does not matter
    b.q[50] = INF
    b.q[103:] = NAN
    sin, out = b.fresh(), b.fresh(11)
    b.run(out, sin, 0.25)
    b.q[3], b.q[50], b.q[103:] = 0, 0, 0                          # the oracle's 0 * NaN is NaN
    b.check(out, sin, 0.25)
    assert (out[1, :, :20] == 0.25 * sin[1, :, :20]).all()


def test_keys_and_rows_that_are_not_finite_stay_where_they_are():
    b = Batch(GQA7, torch.bfloat16, [300], [[40]])
    clean = b.run(torch.zeros_like(b.fresh()))
    k = b.k[0].clone()
    k[0, 7, 0, 5] = NAN
    k[0, 290, 1, :] = INF
    b.bc.update_prefix_layer(b.pid[0], 0, k[0], k[0])
    got = b.run(torch.zeros_like(clean))
    assert torch.isnan(got[0, 0, 7]) and not torch.isfinite(got[0, 1, 290])
    got[0, 0, 7], got[0, 1, 290] = clean[0, 0, 7], clean[0, 1, 290]
    assert torch.equal(got, clean)
    # a key of infinite negative scores: weight 0, also beside rows that add nothing
    b.q.abs_()
    k = b.k[0].clone()
    k[0, 9] = -INF
    b.bc.update_prefix_layer(b.pid[0], 0, k[0], k[0])
    b.lse[5] = INF
    assert (b.run(torch.zeros_like(clean))[0, :, 9] == 0).all()
    b.lse[6, 3] = NAN                                             # a NaN spreads over its KV head
    got = b.run(torch.zeros_like(clean))
    assert torch.isnan(got[0, 0, :300]).all() and torch.isfinite(got[0, 1, :300]).all()


def test_requests_without_a_prefix_are_passed_over():
    b = Batch(MHA, torch.bfloat16, [50, 70], [[4, 5], [6]])
    out, ref = b.fresh(), b.fresh()
    b.run(ref)
    b.bc.prefix_weights(0, [-1] + b.ids[:2] + [-1, -1] + b.ids[2:], [3] + b.off[:2] + [0, 9] + b.off[2:],
                        [9] + b.n[:2] + [0, 2] + b.n[2:], b.q, b.lse, out, [-5] + b.so[:2] + [0, 1] + b.so[2:], scale=SCALE)
    assert torch.equal(out, ref)
    before = out.clone()
    b.bc.prefix_weights(0, [-1], [0], [4], b.q, b.lse, out, [0], scale=SCALE)
    b.bc.prefix_weights(0, [], [], [], b.q, b.lse, out, [], scale=SCALE)
    assert torch.equal(out, before)


def test_many_rows_over_few_keys_are_split_and_repeat_bit_for_bit():
    b = Batch(GQA7, torch.bfloat16, [40], [[700, 900, 33]])
    launches = b.bc.launch_count()
    first = b.run(b.fresh())
    assert b.bc.launch_count() == launches + 2                    # ranges of rows, and their sums
    b.check(first)
    for _ in range(3):
        assert torch.equal(b.run(b.fresh()), first)


def test_more_requests_and_pages_than_one_launch_takes():
    n = [(7 * i) % 3 for i in range(2500)]                        # 2500 row runs, a third of them empty
    b = Batch((2, 1, 128), torch.bfloat16, [33], [n])
    sin, out = b.fresh(), b.fresh(3)
    b.check(b.run(out, sin, 0.5), sin, 0.5)
    b = Batch((1, 1, 128), torch.bfloat16, [16 * 8000 + 5, 100], [[20, 1], [9]])
    launches = b.bc.launch_count()
    sin = b.fresh()
    b.check(b.run(out := b.fresh(3), sin, 1.0), sin, 1.0)
    assert b.bc.launch_count() >= launches + 2
    # both at once: the parts of the rows are added on in launches of their own
    b = Batch((1, 1, 128), torch.bfloat16, [16 * 4200 + 1], [n])
    sin = b.fresh()
    b.check(b.run(out := b.fresh(3), sin, 0.5), sin, 0.5)


def test_rows_past_32_bit_offsets():
    hq, hkv, d, stride, rows = 2, 1, 128, 1 << 22, 700            # the last rows start 2.9 G elements into q
    b = Batch((hq, hkv, d), torch.bfloat16, [90], [[rows]])
    small = b.q.clone()
    big = torch.empty(stride * (rows - 1) + hq * d, dtype=torch.bfloat16, device="cuda")
    b.q = big.as_strided((rows, hq, d), (stride, d, 1))
    b.q.copy_(small[:rows])
    b.lse = b.lse[:rows].contiguous()
    out = b.run(b.fresh())
    b.q = small
    b.lse = torch.cat([b.lse, b.lse[:3]])
    b.check(out)


def test_weights_of_real_attention_sum_to_one_per_row_and_head():
    """lse from attend: the cached keys' weights plus the request's own are 1 for every row and head."""
    b = Batch(GQA7, torch.bfloat16, [1100], [[16, 7]], layers=2)
    k = randn((b.rows, b.hkv, b.d), 1, torch.bfloat16)
    out = torch.empty_like(b.q)
    lse = torch.full((b.rows, b.hq), INF, dtype=torch.float32, device="cuda")     # rows of no request stay so
    for layer in range(2):
        b.bc.attend(layer, b.ids, b.off, b.n, b.q, k, k, out, lse, SCALE)
        b.lse = lse
        w = b.run(b.fresh(), layer=layer)
        b.check(w, layer=layer)
        own = 0.0
        for o, n in zip(b.off, b.n):
            own = own + op.prefix_weights(f64(k)[o:o + n], f64(b.q)[o:o + n], f64(lse)[o:o + n], b.g, SCALE).sum(1)
        total = f64(w)[0, :, :1100].sum(1) + own
        # attend's lse is good to 1e-3 in the tests of attention; a weight moves by as much, relatively
        np.testing.assert_allclose(total, sum(b.n) * b.g, rtol=1e-3)


def test_weights_in_a_graph_on_another_stream_and_after_a_give_up():
    b = Batch(GQA7, torch.bfloat16, [700, 33], [[60, 5], [17]])
    ref = b.run(b.fresh())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = b.fresh(4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):                    # no run before the capture
        b.run(out, out, 0.5)
    start = out.clone()
    torch.cuda.synchronize()
    for i in range(3):
        graph.replay()
    torch.cuda.synchronize()
    want = start.double()
    for _ in range(3):
        want = 0.5 * want + ref.double()
    for i, m in enumerate(b.m):
        torch.testing.assert_close(out[i, :, :m].double(), want[i, :, :m], rtol=8 * 2.0 ** -24, atol=0)
    b.q.mul_(0.5)                                                 # the graph reads the tensors' new contents
    out.copy_(start)
    graph.replay()
    direct = b.run(start.clone(), start, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(out, direct)
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        other = b.run(start.clone(), start, 0.5)
    side.synchronize()
    assert torch.equal(other, direct)
    # a wait budget that ordinary waits exceed: the status says so, and the context works again once cleared
    b.bc.set_wait_budget(1)
    b.run(b.fresh())
    assert b.bc.device_status() == binding.ERR_TIMEOUT
    b.bc.set_wait_budget(0)
    assert b.bc.device_status(clear=True) == binding.ERR_TIMEOUT
    assert torch.equal(b.run(start.clone(), start, 0.5), direct)


# ---------------------------------------------------------------------------------------------
# choice of tokens
# ---------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def bc():
    return binding.BiCache(1, 2, 1, 128, 8, torch.bfloat16, 16, 1)


def select(bc, scores, keep, first=0, last=0):
    idx = torch.full((scores.shape[0], keep + 3), -7, dtype=torch.int32, device="cuda")
    bc.select_tokens(scores, keep, idx[:, :keep], first, last)
    assert (idx[:, keep:] == -7).all()
    return idx[:, :keep].cpu().tolist()


def check_select(bc, scores, keep, first=0, last=0):
    got = select(bc, scores, keep, first, last)
    for r, row in enumerate(scores.cpu().tolist()):
        assert got[r] == op.select_tokens(row, keep, first, last), (r, keep, first, last)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 1023, 1024, 1025, 2049, 5000])
def test_select(bc, n):
    rng = np.random.default_rng(n)
    wide = torch.randn((3, n + 1), generator=gen(n), device="cuda")
    for keep in sorted({1, 2, n // 3 + 1, n - 1, n} & set(range(1, n + 1))):
        check_select(bc, wide[:, 1:], keep)                       # rows that start off any alignment
        check_select(bc, torch.round(wide[:, :n]), keep)          # many ties
        f = int(rng.integers(0, keep + 1))
        check_select(bc, torch.round(wide[:, :n] * 2), keep, f, keep - f if rng.random() < 0.5 else 0)
        check_select(bc, wide[:, :n].exp() * 1e-3, keep, min(1, keep), 0)


def test_select_special_values(bc):
    vals = [NAN, INF, -INF, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0, -1.0, -NAN]
    rng = np.random.default_rng(0)
    x = torch.tensor(rng.choice(vals, size=(6, 700)), dtype=torch.float32, device="cuda")
    for keep in (1, 50, 333, 699, 700):
        check_select(bc, x, keep)
        check_select(bc, x, keep, min(keep, 20), min(10, max(0, keep - 20)))
    for v in vals:                                                # a row of one value
        check_select(bc, torch.full((2, 321), v, device="cuda"), 100, 3, 5)
    assert select(bc, x[:, :30], 30, 900, 900) == [list(range(30))] * 6
    assert select(bc, x[:0], 5) == [] and select(bc, x, 0) == [[]] * 6


@pytest.mark.parametrize("n", [16384, 40001, 49149, 49150, 49153, 131072, 300007, 393300])
def test_select_long_rows(bc, n):
    x = torch.exp(torch.randn((3, n), generator=gen(n), device="cuda") * 2 - 5)
    x[1] = (x[1] * 64).round()
    x[2, n // 2:] = 0
    for keep, first, last in ((1, 0, 0), (n // 4, 4, 64), (n - 5, 0, 1)):
        got = torch.empty((3, keep), dtype=torch.int32, device="cuda")
        bc.select_tokens(x, keep, got, first, last)
        s = x.double().cpu().numpy()
        prot = np.zeros(n, bool)
        prot[:first] = True
        prot[n - last:] = True
        for r in range(3):
            want = np.sort(np.lexsort((np.arange(n), -s[r], ~prot))[:keep])
            assert np.array_equal(got[r].cpu().numpy(), want)


# ---------------------------------------------------------------------------------------------
# compaction
# ---------------------------------------------------------------------------------------------

def read(bc, pid, layer, m):
    k = torch.empty((m, bc.Hkv, bc.D), dtype=bc.dtype, device="cuda")
    v = torch.empty_like(k)
    bc.read_prefix_layer(pid, layer, k, v)
    return k, v


@pytest.mark.parametrize("dtype,heads,m,keep", [
    (torch.bfloat16, (3, 3, 128), 203, 77), (torch.bfloat16, (2, 1, 128), 16, 16), (torch.bfloat16, (4, 4, 64), 33, 1),
    (torch.float32, (2, 2, 128), 100, 99), (torch.float32, (1, 1, 32), 5, 17), (torch.bfloat16, (2, 2, 96), 50, 31)])
@pytest.mark.parametrize("per_layer_lists", [False, True])
def test_compact(dtype, heads, m, keep, per_layer_lists):
    hq, hkv, d = heads
    L = 3
    pages = (m + 15) // 16 + (keep + 15) // 16 + 4
    bc = binding.BiCache(L, hq, hkv, d, pages, dtype, 16, 1, free_order=workloads.shuffled_page_order(pages, 3),
                         layer_pages=[pages, pages - 1, pages] if per_layer_lists else None)
    k, v = randn((L, m, hkv, d), 1, dtype), randn((L, m, hkv, d), 2, dtype)
    src, _, _ = bc.put_prefix(1, k, v)
    if per_layer_lists:
        bc.reserve_prefix(3, 16, first_layer=1)                   # the layers' free queues part ways
    dst, _, _ = bc.reserve_prefix(2, keep)
    idx = torch.randint(0, m, (L, hkv, keep + 2), generator=gen(4), device="cuda", dtype=torch.int32)[:, :, 1:-1]
    bc.compact_prefix(src, dst, idx)                              # any order, repeats
    for l in range(L):
        gk, gv = read(bc, dst, l, keep)
        for h in range(hkv):
            assert torch.equal(gk[:, h], k[l, idx[l, h].long(), h]) and torch.equal(gv[:, h], v[l, idx[l, h].long(), h])
    one = idx[1:2, :1]
    bc.compact_prefix(src, dst, one, first_layer=2)               # one layer, one list for the heads
    gk, gv = read(bc, dst, 2, keep)
    assert torch.equal(gk, k[2, one[0, 0].long()]) and torch.equal(gv, v[2, one[0, 0].long()])
    gk, _ = read(bc, dst, 1, keep)
    assert torch.equal(gk[:, 0], k[1, idx[1, 0].long(), 0])       # the other layers as they were
    sk, sv = read(bc, src, 1, m)
    assert torch.equal(sk, k[1]) and torch.equal(sv, v[1])
    assert bc.device_status() == 0


def test_an_index_outside_the_source_is_a_zero_token_and_a_status(bc_pages=40):
    bc = binding.BiCache(1, 2, 2, 128, bc_pages, torch.bfloat16, 16, 1)
    k = randn((1, 50, 2, 128), 1, torch.bfloat16)
    src, _, _ = bc.put_prefix(1, k, k)
    dst, _, _ = bc.reserve_prefix(2, 20)
    idx = torch.arange(20, device="cuda", dtype=torch.int32).expand(1, 2, 20).clone()
    for bad in (-1, 50, 2 ** 31 - 1, -2 ** 31):
        idx[0, 1, 3] = bad
        bc.compact_prefix(src, dst, idx)
        assert bc.device_status() == binding.ERR_INVALID
        assert bc.device_status(clear=True) == binding.ERR_INVALID and bc.device_status() == 0
        gk, _ = read(bc, dst, 0, 20)
        assert not gk[3, 1].any()
        gk[3, 1] = k[0, 3, 1]
        assert torch.equal(gk, k[0, :20])


def test_compact_of_more_pages_than_one_launch_takes():
    m, keep = 16 * 6000 + 3, 16 * 2500 + 1
    bc = binding.BiCache(1, 1, 1, 32, 8600, torch.float32, 16, 1, free_order=workloads.shuffled_page_order(8600, 1))
    k = randn((1, m, 1, 32), 1, torch.float32)
    src, _, _ = bc.put_prefix(1, k, -k)
    dst, _, _ = bc.reserve_prefix(2, keep)
    idx = torch.randperm(m, generator=gen(2), device="cuda")[:keep].to(torch.int32)[None, None]
    idx[0, 0, 5] = m                                              # noticed once, whatever the number of launches
    launches = bc.launch_count()
    bc.compact_prefix(src, dst, idx)
    assert bc.launch_count() == launches + 2
    assert bc.device_status(clear=True) == binding.ERR_INVALID
    idx[0, 0, 5] = 0
    gk, gv = read(bc, dst, 0, keep)
    want = k[0, idx[0, 0].long()]
    want[5] = 0
    assert torch.equal(gk, want) and torch.equal(gv, -want)


@pytest.mark.parametrize("pages", [100, 223, 224, 225, 1100, 1216, 1217, 2000, 2432, 2433, 3500])
def test_lists_of_every_length(pages):
    """The page lists travel as launch parameters of several lengths: weights, compaction and read-back around each."""
    b = Batch((2, 1, 128), torch.bfloat16, [16 * pages - 3], [[5]], extra=pages // 2 + 1)
    sin = b.fresh()
    b.check(b.run(out := b.fresh(3), sin, 0.5), sin, 0.5)
    keep = 16 * (pages // 2) + 1
    dst, _, _ = b.bc.reserve_prefix(9, keep)
    idx = torch.randint(0, b.m[0], (1, 1, keep), generator=gen(4), device="cuda", dtype=torch.int32)
    b.bc.compact_prefix(b.pid[0], dst, idx)
    for pid, m, want in ((dst, keep, b.k[0][0, idx[0, 0].long()]), (b.pid[0], b.m[0], b.k[0][0])):
        gk, gv = read(b.bc, pid, 0, m)
        assert torch.equal(gk, want) and torch.equal(gv, -want)
    assert b.bc.device_status() == 0


# ---------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,heads,tol", [(torch.bfloat16, GQA7, 2e-2), (torch.float32, (4, 2, 64), 1e-4)])
def test_attend_weigh_choose_shorten_attend(dtype, heads, tol):
    """Two layers: attend over the whole prefix, accumulate the weights over two steps, keep half of the tokens
    per KV head, and attend over the shortened prefix; attention over the kept keys against the oracle."""
    m, keep, L = 1200, 600, 2
    b = Batch(heads, dtype, [m], [[9, 14]], layers=L, extra=(keep + 15) // 16)
    k = randn((b.rows, b.hkv, b.d), 1, dtype)
    out = torch.zeros_like(b.q)
    lse = torch.full((b.rows, b.hq), INF, dtype=torch.float32, device="cuda")
    scores = torch.empty((L, b.hkv, m), device="cuda")
    for step in range(2):
        for l in range(L):
            b.bc.attend(l, b.ids, b.off, b.n, b.q, k, k, out, lse, SCALE)
            b.bc.prefix_weights(l, b.ids, b.off, b.n, b.q, lse, scores[l:l + 1], [0, 0],
                                scores_in=scores[l:l + 1] if step else None, decay=float(step), scale=SCALE)
    idx = torch.empty((L, b.hkv, keep), dtype=torch.int32, device="cuda")
    b.bc.select_tokens(scores.view(L * b.hkv, m), keep, idx.view(L * b.hkv, keep), 4, 32)
    short, _, _ = b.bc.reserve_prefix(500, keep)
    b.bc.compact_prefix(b.pid[0], short, idx)
    assert b.bc.device_status() == 0
    for r, row in enumerate(scores.view(L * b.hkv, m).cpu().tolist()):
        assert idx.view(-1, keep)[r].cpu().tolist() == op.select_tokens(row, keep, 4, 32)
    for l in range(L):
        b.bc.attend(l, [short, short], b.off, b.n, b.q, k, k, out, lse, SCALE)
        got = f64(out)
        st = oracle.PagedPrefixStore(1, b.hkv, b.d, 16, (keep + 15) // 16)
        kept = torch.stack([b.k[0][l, idx[l, h].long(), h] for h in range(b.hkv)], 1)
        opid, _, _ = st.put(1, f64(kept)[None], -f64(kept)[None])
        ref, _ = oracle.attend(st, 0, [opid, opid], b.off, b.n, f64(b.q), f64(k), f64(k), SCALE)
        rows = sum(b.n)
        assert np.abs(got[:rows] - ref[:rows]).max() <= tol


def test_choice_and_compaction_in_a_graph():
    b = Batch(MHA, torch.bfloat16, [100], [[20]], extra=4)
    short, _, _ = b.bc.reserve_prefix(9, 50)
    scores, idx = b.fresh(), torch.zeros((1, b.hkv, 50), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.run(scores)
        b.bc.select_tokens(scores[0, :, :100], 50, idx[0], 1, 1)
        b.bc.compact_prefix(b.pid[0], short, idx)
    for step in range(2):
        b.q.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        ref = b.run(b.fresh())
        for h in range(b.hkv):
            assert idx[0, h].cpu().tolist() == op.select_tokens(ref[0, h, :100].cpu().tolist(), 50, 1, 1)
        gk, gv = read(b.bc, short, 0, 50)
        for h in range(b.hkv):
            assert torch.equal(gk[:, h], b.k[0][0, idx[0, h].long(), h]) and torch.equal(gv[:, h], -gk[:, h])

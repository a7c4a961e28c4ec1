"""GPU parity of windowed attention over cached tokens against the fp64 oracle.

Tolerance.  A = scale * sum |q||k| of the largest visible score.  A score is D products added in fp32 (the tensor cores
may truncate: a whole unit, 2^-23, each), scaled and brought to the exponent in a few roundings more: off by at most
(D + 8) 2^-23 A; the exponential by 2^-20 relative.  So a weight is off by e = (D + 8) 2^-23 A + 2^-20 relative, before and
after division by their sum: 2 e; sums over K keys add K / 16 + 64 steps of 2^-23.  On the tensor cores weights are
rounded to bf16, half a step, 2^-8, before they meet the values.  All this is relative to sum w |v|.  The output is rounded once,
half a step.  The log-sum-exp: e and the steps of the sum, plus 2^-22 of its value for logarithm and reference."""
import math

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


def randn(shape, seed, dtype, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


HEADS = {"mha32": (32, 32, 128), "gqa32": (32, 8, 128), "gqa7": (7, 1, 128), "gqa4": (8, 2, 128), "gqa28": (28, 4, 128), "mha2": (2, 2, 128), "gqa150": (150, 1, 128),
         "mha4_64": (4, 4, 64), "gqa2_96": (2, 1, 96), "d256": (3, 1, 256), "d32": (2, 2, 32)}


class Batch:
    """Prefixes of given lengths (reserved `spare` tokens longer, everything behind the cached tokens NaN), requests with
    rows in between which others lie."""

    def __init__(self, heads, dtype, lens, requests, spare=0, std=1.5, path=None, shuffled=True):
        self.hq, self.hkv, self.d = HEADS[heads]
        self.dtype, self.lens, self.requests = dtype, lens, requests         # request: prefix index, position, rows
        pages = sum((m + spare + 15) // 16 for m in lens) + 1
        order = np.random.default_rng(1).permutation(pages)
        self.rows = sum(n for _, _, n in requests) + len(requests) + 1
        self.bc = binding.BiCache(1, self.hq, self.hkv, self.d, pages, dtype, self.rows, len(requests),
                                  free_order=order if shuffled else None)
        self.bc.k_pool.fill_(255)
        self.bc.v_pool.fill_(255)
        if path is not None:
            self.bc.set_path(path)
        self.ids, self.k, self.v = [], [], []
        for i, m in enumerate(lens):
            pid = self.bc.reserve_prefix(i + 1, max(1, m + spare))[0]
            k, v = randn((m, self.hkv, self.d), 10 * i + 1, dtype), randn((m, self.hkv, self.d), 10 * i + 2, dtype)
            if m:
                self.bc.append_tokens(0, [pid], [0], [0], [m], k, v)
            self.ids.append(pid)
            self.k.append(k)
            self.v.append(v)
        self.q = randn((self.rows, self.hq + 1, self.d), 5, dtype, std)[:, :self.hq]
        self.off, at = [], 1
        for _, _, n in requests:
            self.off.append(at)
            at += n + 1

    def call(self, sinks, left, right, scale=None, out=None, lse="new"):
        out = torch.full((self.rows, self.hq, self.d), 9.0, dtype=self.dtype, device="cuda") if out is None else out
        lse = torch.full((self.rows, self.hq), 9.0, device="cuda") if isinstance(lse, str) else lse
        r = self.requests
        self.bc.attend_window(0, [self.ids[i] for i, _, _ in r], [self.lens[i] for i, _, _ in r], [p for _, p, _ in r],
                              self.off, [n for _, _, n in r], self.q, out, lse, sinks, left, right, scale)
        return out, lse

    def check(self, sinks, left, right, scale=None, weights_bf16=None):
        out, lse = self.call(sinks, left, right, scale)
        assert self.bc.device_status() == 0
        scale = self.d ** -0.5 if scale is None else scale
        tensor = self.bc.last_attention_kernel() != binding.KERNEL_SIMT
        assert weights_bf16 is None or tensor == weights_bf16
        mine = np.zeros(self.rows, dtype=bool)
        for (i, p, n), o in zip(self.requests, self.off):
            mine[o:o + n] = True
            if n == 0:
                continue
            ref, rl, mag, size = gc.attend_window(f64(self.q[o:o + n]), f64(self.k[i]), f64(self.v[i]), p, sinks, left, right, scale)
            steps = (self.lens[i] / 16 + 64) * 2.0 ** -23
            e = (self.d + 8) * 2.0 ** -23 * abs(size) + 2.0 ** -20
            tol = mag * ((2.0 ** -8 if tensor else 0) + 2 * e + steps)[..., None]
            tol = tol + (np.abs(ref) + tol) * torch.finfo(self.dtype).eps / 2
            err = np.abs(f64(out[o:o + n]) - ref)
            assert (err <= tol).all(), (i, p, n, np.nanmax(err - tol), np.unravel_index(np.nanargmax(err - tol), err.shape))
            got = f64(lse[o:o + n])
            none = np.isneginf(rl)
            assert (np.isneginf(got) == none).all() and not f64(out[o:o + n])[none].any()
            # the reference of the running maximum is at most 2^8 below the scores: its own size is the score's
            assert (np.abs(got[~none] - rl[~none]) <= (e + steps + 2.0 ** -22 * (np.abs(rl) + size + 8))[~none]).all()
        assert (out[torch.tensor(~mine)] == 9).all() and (lse[torch.tensor(~mine)] == 9).all()
        return out, lse


WINDOWS = [(0, -1, -1), (0, -1, 0), (4, 100, 0), (0, 0, 0), (17, 33, 5), (129, 64, -1), (1000, 10, 0), (0, 5, -1), (1, 300, 129),
           (64, 63, 0)]
LENS = [0, 1, 15, 16, 17, 63, 64, 65, 128, 200, 300, 1000]
# rows at the end of the cache, at its start, past it by less and by more than windows reach; blocks and single tokens
REQUESTS = ([(i, max(0, m - n), n) for i, m in enumerate(LENS) for n in (1, 5)] +
            [(11, 0, 40), (11, 500, 70), (11, 1000, 3), (11, 1090, 20), (10, 5000, 2), (9, 190, 0), (7, 40, 30), (11, 990, 10),
             (8, 0, 128), (10, 290, 33)])


@pytest.mark.parametrize("window", WINDOWS)
@pytest.mark.parametrize("heads,dtype", [("gqa7", torch.bfloat16), ("gqa4", torch.bfloat16), ("gqa150", torch.bfloat16),
                                         ("mha4_64", torch.float32), ("gqa2_96", torch.float32), ("d256", torch.bfloat16),
                                         ("d32", torch.bfloat16), ("mha2", torch.float32)])
def test_ragged(window, heads, dtype):
    Batch(heads, dtype, LENS, REQUESTS, spare=21).check(*window)


@pytest.mark.parametrize("window", WINDOWS[1:6])
def test_ragged_on_cuda_cores(window):
    Batch("gqa4", torch.bfloat16, LENS, REQUESTS, spare=21, path=binding.PATH_SIMT).check(*window, weights_bf16=False)


@pytest.mark.parametrize("window", [(0, -1, 0), (4, 700, 0), (0, 127, 128), (0, 300, -1), (33, 64, 17)])
@pytest.mark.parametrize("heads,dtype", [("gqa7", torch.bfloat16), ("mha2", torch.bfloat16), ("gqa4", torch.bfloat16),
                                         ("mha4_64", torch.float32)])
def test_prompts(window, heads, dtype):
    lens = [700, 1531, 257]
    Batch(heads, dtype, lens, [(0, 0, 700), (1, 400, 1131), (2, 0, 256), (1, 1600, 130)]).check(*window)


@pytest.mark.parametrize("window", [(0, -1, 0), (4, 700, 0), (0, 127, 128), (0, 300, -1), (33, 64, 17), (0, 0, 0), (129, 200, 0)])
@pytest.mark.parametrize("heads", ["gqa28", "mha32", "gqa32", "gqa150"])
def test_row_tiles_of_256(window, heads):
    """Enough rows for the kernel with row tiles of 256: prompts, rows that see nothing, an empty cache, a few rows."""
    lens = [700, 901, 257, 0]
    requests = [(0, 0, 700), (1, 400, 501), (2, 0, 256), (1, 1300, 130), (3, 5, 200), (0, 699, 1), (2, 200, 40), (1, 880, 129)]
    b = Batch(heads, torch.bfloat16, lens, requests * 2, spare=37)
    out, _ = b.check(*window)
    by_256 = 128 % (b.hq // b.hkv) == 0                        # else tiles of 128 rows
    assert b.bc.last_attention_kernel() == (binding.KERNEL_TENSOR if by_256 else binding.KERNEL_KEY_RANGES)
    again, _ = b.call(*window)
    assert torch.equal(out, again)


def test_unseen_tokens_and_row_tiles_of_256():
    m, n, sinks, left = 2600, 1500, 5, 70
    b = Batch("gqa32", torch.bfloat16, [m], [(0, m - n, n)] * 3)
    want = b.call(sinks, left, 0)
    assert b.bc.last_attention_kernel() == binding.KERNEL_TENSOR
    first = m - n - left
    bad = torch.full((first - sinks, b.hkv, b.d), math.nan, dtype=torch.bfloat16, device="cuda")
    b.bc.append_tokens(0, [b.ids[0]], [sinks], [0], [first - sinks], bad, -bad * math.inf)
    got = b.call(sinks, left, 0)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and want[0].isfinite().all()


@pytest.mark.parametrize("m", [1023, 4096, 20000])
@pytest.mark.parametrize("heads,dtype", [("gqa28", torch.bfloat16), ("mha2", torch.bfloat16), ("mha4_64", torch.float32),
                                         ("gqa2_96", torch.float32)])
@pytest.mark.parametrize("n", [1, 16])
def test_few_rows_against_many_keys(m, heads, dtype, n):
    b = Batch(heads, dtype, [m], [(0, m - n, n)])
    before = b.bc.launch_count()
    out, lse = b.check(0, -1, 0)
    assert b.bc.launch_count() - before == 2                   # ranges of keys, and their join
    again, _ = b.call(0, -1, 0)
    assert torch.equal(out, again)
    b.check(4, m // 2, 0)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = np.random.default_rng(seed)
    heads = ["gqa7", "gqa4", "mha2", "mha32", "mha4_64", "d32"][seed % 6]
    dtype = torch.float32 if heads == "mha4_64" else torch.bfloat16
    lens = [int(x) for x in np.exp(rng.uniform(0, math.log(2500), rng.integers(1, 5)))]
    most = 700 if heads == "mha32" else 300
    requests = []
    for _ in range(rng.integers(1, 9)):
        i = int(rng.integers(0, len(lens)))
        n = int(rng.choice([1, rng.integers(1, 20), rng.integers(1, most)]))
        requests.append((i, int(rng.choice([max(0, lens[i] - n), rng.integers(0, lens[i] + 50)])), n))
    window = (int(rng.choice([0, 1, 4, rng.integers(0, 300)])), int(rng.choice([-1, 0, rng.integers(0, 900)])),
              int(rng.choice([-1, 0, rng.integers(0, 200)])))
    Batch(heads, dtype, lens, requests, spare=int(rng.integers(0, 40)), shuffled=bool(seed % 4)).check(*window)


def test_split_and_whole_requests_in_one_call():
    lens = [20000, 40, 9000, 17]
    Batch("gqa28", torch.bfloat16, lens, [(1, 39, 1), (0, 19999, 1), (3, 3, 14), (2, 8990, 10), (1, 0, 16)]).check(2, -1, 0)


@pytest.mark.parametrize("heads,dtype", [("gqa4", torch.bfloat16), ("mha4_64", torch.float32)])
@pytest.mark.parametrize("n", [3, 300])
def test_unseen_tokens_may_hold_anything(heads, dtype, n):
    m, sinks, left = 900, 5, 70
    b = Batch(heads, dtype, [m], [(0, m - n, n)])
    want = b.call(sinks, left, 0)
    first = m - n - left
    bad_k, bad_v = randn((first - sinks, b.hkv, b.d), 1, dtype), randn((first - sinks, b.hkv, b.d), 2, dtype)
    bad_k[::2], bad_k[1::2], bad_v[::2], bad_v[1::2] = math.nan, math.inf, -math.inf, math.nan
    b.bc.append_tokens(0, [b.ids[0]], [sinks], [0], [first - sinks], bad_k, bad_v)
    got = b.call(sinks, left, 0)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and want[0].isfinite().all()


@pytest.mark.parametrize("heads,dtype", [("gqa4", torch.bfloat16), ("mha4_64", torch.float32)])
@pytest.mark.parametrize("n", [3, 300])
def test_a_nan_that_is_seen_spreads(heads, dtype, n):
    b = Batch(heads, dtype, [800], [(0, 800 - n, n)])
    b.bc.append_tokens(0, [b.ids[0]], [799], [0], [1], torch.full((1, b.hkv, b.d), math.nan, dtype=dtype, device="cuda"),
                       b.v[0][799:])
    out, lse = b.call(0, -1, 0)
    rows = slice(b.off[0], b.off[0] + n)
    assert out[rows][-1].isnan().all() and lse[rows][-1].isnan().all()       # the last row sees the last key
    assert out[rows][:-1].isfinite().all() and lse[rows][:-1].isfinite().all()


@pytest.mark.parametrize("heads,dtype,many", [("gqa4", torch.bfloat16, False), ("gqa32", torch.bfloat16, True), ("mha4_64", torch.float32, False)])
def test_steep_scores(heads, dtype, many):
    """Scores that grow along the keys by far more than the running reference follows at a time."""
    b = Batch(heads, dtype, [700], [(0, 690, 10), (0, 0, 300)] * (12 if many else 1), std=0.1)
    ramp = torch.linspace(-30, 30, 700, device="cuda")[:, None, None]
    k = (torch.ones((700, b.hkv, b.d), device="cuda") * ramp).to(dtype)
    b.q[...] = 0.25
    b.k[0] = k
    b.bc.append_tokens(0, b.ids, [0], [0], [700], k, b.v[0])
    for w in ((0, -1, -1), (3, 100, 0), (0, 40, 40)):
        b.check(*w)
    b.k[0] = k.flip(0)
    b.bc.append_tokens(0, b.ids, [0], [0], [700], b.k[0], b.v[0])
    for w in ((0, -1, -1), (3, 100, 0), (0, 40, 40)):
        b.check(*w)


@pytest.mark.parametrize("scale", [0.0, -0.05, 0.3])
def test_scales(scale):
    Batch("gqa4", torch.bfloat16, [300], [(0, 200, 100), (0, 299, 1)]).check(3, 150, 0, scale)


def test_strided_rows_no_lse_and_shared_prefixes():
    b = Batch("gqa4", torch.bfloat16, [500], [(0, 100, 7), (0, 480, 20), (0, 100, 7)])
    want, _ = b.check(4, 64, 0)
    wide = torch.full((b.rows, b.hq + 3, b.d), 9.0, dtype=torch.bfloat16, device="cuda")
    b.call(4, 64, 0, out=wide[:, :b.hq], lse=None)
    assert torch.equal(wide[:, :b.hq], want) and (wide[:, b.hq:] == 9).all()


def test_pages_that_do_not_fit_the_parameters():
    """A request with more pages than a launch's parameters hold, between others."""
    m = 130000
    b = Batch("d32", torch.bfloat16, [m, 100], [(1, 90, 10), (0, m - 3, 3), (1, 99, 1)])
    b.check(0, -1, 0)
    b.check(7, 127500, 0)


@pytest.mark.parametrize("heads,dtype", [("gqa28", torch.bfloat16), ("mha32", torch.bfloat16), ("mha4_64", torch.float32)])
@pytest.mark.parametrize("window", [(0, -1, 0), (20, 200, 30)])
def test_consecutive_and_shuffled_pages_give_the_same_bits(heads, dtype, window):
    lens = [700, 3001, 17, 0]
    requests = [(0, 100, 300), (1, 3000, 1), (2, 16, 5), (1, 900, 700), (3, 0, 2), (0, 650, 50), (1, 1300, 900)]
    outs = [Batch(heads, dtype, lens, requests, spare=5, shuffled=s).call(*window) for s in (False, True)]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    Batch(heads, dtype, lens, requests[:3], spare=5, shuffled=False).check(*window)


def test_long_lists_go_through_the_workspace():
    """Page lists of a batch that together do not fit the parameters: launches that write them, then one and a join."""
    lens = [20000, 30000, 40000, 50000]
    b = Batch("d32", torch.bfloat16, lens, [(i, m - 2, 2) for i, m in enumerate(lens)])
    before = b.bc.launch_count()
    b.check(4, -1, 0)
    assert b.bc.launch_count() - before == 4                   # 8750 pages: two lists
    b.check(4, 25000, 0)


def test_many_requests_take_several_launches():
    lens = [1 + 37 * i % 400 for i in range(300)]
    b = Batch("d32", torch.bfloat16, lens, [(i, max(0, m - 2), 1 + i % 3) for i, m in enumerate(lens)] * 3)
    before = b.bc.launch_count()
    b.check(2, 60, 0)
    assert b.bc.launch_count() - before >= 2


def test_another_stream_and_device_guard():
    b = Batch("gqa4", torch.bfloat16, [5000], [(0, 4990, 10)])
    want, wl = b.call(0, -1, 0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, gl = b.call(0, -1, 0)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(gl, wl)


@pytest.mark.parametrize("window", [(0, 2 ** 31 - 1, 0), (5, 40, 2 ** 31 - 1), (2 ** 31 - 1, 3, 0), (0, 2 ** 31 - 1, 2 ** 31 - 1), (7, 2 ** 31 - 1, 90)])
@pytest.mark.parametrize("heads,dtype", [("gqa4", torch.bfloat16), ("gqa7", torch.bfloat16), ("mha4_64", torch.float32)])
def test_windows_and_positions_at_the_end_of_their_range(window, heads, dtype):
    """Sums of two of them do not fit 32 bits: a window as wide as numbers go is one without bound, and the last row
    that has a position stands at 2^31 - 2."""
    top = 2 ** 31 - 1
    Batch(heads, dtype, [0, 100, 700], [(2, 0, 90), (2, 600, 100), (2, top - 90, 90), (1, top - 1, 1), (0, top - 4, 4), (1, 99, 1)]).check(*window)


@pytest.mark.parametrize("window", [(0, 2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1, 0)])
def test_row_tiles_of_256_at_the_end_of_their_range(window):
    b = Batch("mha32", torch.bfloat16, [300], [(0, 2 ** 31 - 1 - 4000, 4000), (0, 100, 200)])
    b.check(*window)
    assert b.bc.last_attention_kernel() == binding.KERNEL_TENSOR

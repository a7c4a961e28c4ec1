"""Wait budgets shorter than what the kernels wait for, but not the strictest one, which gives up before any work: a role may
give up while the others still work and copies are under way.  (A wait asks the hardware first, which itself waits a
while: waits of a few microseconds end before the budget counts, those for a whole item run out.)  Whatever happens the call
ends with its copies landed: a call of another context, which follows at once and may be placed on the same SMs, has the
right bits; the status says what happened; a call whose waits did not run out is right; and the context works
again."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
BUDGETS = [1024, 1500, 2500, 4000, 7000, 12000, 20000, 40000]         # SM cycles


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def randn(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def give_up(make, call):
    """make(): a context and what its calls need; call(context, ...): the outputs of one call.  How many calls gave up."""
    (bc, *args), (other, *other_args) = make(), make()
    want = call(bc, *args)
    assert bc.device_status() == binding.OK
    for a, b in zip(want, call(other, *other_args)):
        assert torch.equal(a, b)
    gave_up = 0
    for budget in BUDGETS * 3:
        bc.set_wait_budget(budget)
        first = call(bc, *args)
        after = call(other, *other_args)
        status = bc.device_status(clear=True)
        assert status in (binding.OK, binding.ERR_TIMEOUT) and other.device_status() == binding.OK
        for a, b in zip(want, after):
            assert torch.equal(a, b)
        gave_up += status != binding.OK
        if status == binding.OK:
            for a, b in zip(want, first):
                assert torch.equal(a, b)
    bc.set_wait_budget(0)
    for a, b in zip(want, call(bc, *args)):
        assert torch.equal(a, b)
    assert bc.device_status() == binding.OK
    bc.close()
    other.close()
    return gave_up


# heads, cached tokens, rows, window, kernel: items of many tiles, ranges of keys and their join; items of no more tiles
# than there are slots for
WINDOWS = [(14, 2, 20000, 5, (4, 10000, 0), binding.KERNEL_KEY_RANGES), (32, 32, 700, 300, (4, 350, 0), binding.KERNEL_KEY_RANGES),
           (28, 4, 1500, 1500, (0, 20, 0), binding.KERNEL_KEY_RANGES), (4, 4, 60, 40, (0, -1, -1), binding.KERNEL_KEY_RANGES),
           (32, 32, 3500, 3500, (4, 1750, 0), binding.KERNEL_TENSOR), (8, 8, 15000, 15000, (0, -1, -1), binding.KERNEL_TENSOR)]


@pytest.mark.parametrize("hq,hkv,m,n,window,kernel", WINDOWS)
def test_windowed_attention(hq, hkv, m, n, window, kernel):
    k, q = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2)

    def make():
        bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, 1)
        return bc, bc.put_prefix(1, k, k.flip(1))[0]

    def call(bc, pid):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        bc.attend_window(0, [pid], [m], [m - n], [0], [n], q, out, lse, *window)
        assert bc.last_attention_kernel() == kernel
        return out, lse
    assert give_up(make, call) or m < 10000 or kernel != binding.KERNEL_TENSOR       # items of 100 us: some waits run out


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("hq,hkv,m,lens", [(32, 8, 500, [700, 130, 256, 513, 64, 900]), (8, 8, 1200, [12000]), (14, 2, 300, [40, 7, 333])])
def test_attention(hq, hkv, m, lens, full):
    """Row tiles of one and of several requests; items that take long, and that are split."""
    n = sum(lens)
    off = [sum(lens[:i]) for i in range(len(lens))]
    pk, q, k, v = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)

    def make():
        bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, len(lens))
        bc.set_path(binding.PATH_TENSOR)
        return bc, bc.put_prefix(1, pk, -pk)[0]

    def call(bc, pid):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        if full:
            bc.attend_full(0, off, lens, q, k, v, out, lse)
        else:
            bc.attend(0, [pid] * len(lens), off, lens, q, k, v, out, lse)
        assert bc.last_attention_kernel() == binding.KERNEL_TENSOR
        return out, lse
    assert give_up(make, call) or lens != [12000]


@pytest.mark.parametrize("hq,hkv,m,lens", [(28, 4, 16384, [16]), (4, 4, 2000, [7, 12]), (32, 8, 5000, [1] * 30)])
def test_few_rows_against_a_long_prefix(hq, hkv, m, lens):
    n = sum(lens)
    off = [sum(lens[:i]) for i in range(len(lens))]
    pk, q, k, v = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)

    def make():
        bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, len(lens))
        return bc, bc.put_prefix(1, pk, -pk)[0]

    def call(bc, pid):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        bc.attend(0, [pid] * len(lens), off, lens, q, k, v, out, lse)
        assert bc.last_attention_kernel() == binding.KERNEL_KEY_RANGES
        return out, lse
    give_up(make, call)


@pytest.mark.parametrize("hq,hkv,m,lens", [(28, 4, 4000, [2048]), (4, 4, 300, [40, 7, 3000]), (14, 2, 16384, [16])])
def test_accumulated_weights(hq, hkv, m, lens):
    """Rows by boxes and gathered, items of many row tiles and of few."""
    n = sum(lens) + len(lens)
    off = [sum(lens[:i]) + i for i in range(len(lens))]          # a row between two requests
    pk, q = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2)
    lse = torch.full((n, hq), 5.0, device="cuda")

    def make():
        bc = binding.BiCache(1, hq, hkv, 128, (m + 15) // 16, torch.bfloat16, n, len(lens))
        return bc, bc.put_prefix(1, pk, -pk)[0]

    def call(bc, pid):
        scores = torch.zeros((hkv, m), device="cuda")
        bc.prefix_weights(0, [pid] * len(lens), off, lens, q, lse, scores, [0] * len(lens))
        return scores,
    give_up(make, call)


@pytest.mark.parametrize("hkv,m,d_model", [(4, 700, 512), (1, 256, 64), (8, 20000, 4096)])
@pytest.mark.parametrize("rotated", [False, True])
def test_projection(hkv, m, d_model, rotated):
    """CTAs in pairs: fewer K steps than stages, and many tiles to a pair."""
    h, w_k, w_v = workloads.draw_hidden_and_weights(m, d_model, hkv, 128, 9, device="cuda")
    table = torch.rand((m, 64, 2), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") if rotated else None

    def make():
        bc = binding.BiCache(1, hkv, hkv, 128, (m + 15) // 16, torch.bfloat16, 16, 1)
        return bc, bc.reserve_prefix(1, m)[0]

    def call(bc, pid):
        bc.project_prefix_layer(pid, 0, h, w_k, w_v, table)
        k, v = torch.zeros((m, hkv, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, hkv, 128), dtype=torch.bfloat16, device="cuda")
        bc.read_prefix_layer(pid, 0, k, v)
        return k, v
    give_up(make, call)


@pytest.mark.parametrize("hq,hkv,lens", [(4, 4, [300, 517]), (28, 4, [1000]), (8, 8, [12000])])
def test_attention_on_pairs(hq, hkv, lens):
    n = sum(lens)
    off = [sum(lens[:i]) for i in range(len(lens))]
    q, k, v = randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)

    def make():
        bc = binding.BiCache(1, hq, hkv, 128, 4, torch.bfloat16, n, len(lens))
        bc.set_path(binding.PATH_TENSOR_PAIRS)
        return bc, None

    def call(bc, _):
        out, lse = torch.zeros_like(q), torch.zeros((n, hq), device="cuda")
        bc.attend_full(0, off, lens, q, k, v, out, lse)
        assert bc.last_attention_kernel() == binding.KERNEL_TENSOR_PAIRS
        return out, lse
    assert give_up(make, call) or lens != [12000]


def test_no_wait_runs_out_in_ordinary_calls():
    """The load warps' waits at the end of a block name the last use of every slot, whichever way its tile came (bulk copies,
    boxes, gathered rows): calls of 10 to 200 us take no milliseconds, which a wait that cannot end would."""
    hq, hkv, m = 28, 4, 2000
    lens = [333, 1, 700, 16]
    n, off = sum(lens), [0, 333, 334, 1034]
    pk, q, k, v = randn((1, m, hkv, 128), 1), randn((n, hq, 128), 2), randn((n, hkv, 128), 3), randn((n, hkv, 128), 4)
    bc = binding.BiCache(1, hq, hkv, 128, 126, torch.bfloat16, n, 4)
    pid = bc.put_prefix(1, pk, -pk)[0]
    out, lse, scores = torch.empty_like(q), torch.full((n, hq), 5.0, device="cuda"), torch.empty((hkv, m), device="cuda")
    h, w_k, w_v = workloads.draw_hidden_and_weights(m, 512, hkv, 128, 9, device="cuda")
    short = bc.reserve_prefix(2, 16)[0]

    def paths(path, call):
        def f():
            bc.set_path(path)
            call()
            bc.set_path(binding.PATH_AUTO)
        return f
    for call in (lambda: bc.attend(0, [pid] * 4, off, lens, q, k, v, out), lambda: bc.attend(0, [-1, pid], [0, 333], [100, 1], q, k, v, out),
                 lambda: bc.attend(0, [pid], [1034], [16], q, k, v, out), lambda: bc.attend_full(0, off, lens, q, k, v, out),
                 paths(binding.PATH_TENSOR_PAIRS, lambda: bc.attend_full(0, off, lens, q, k, v, out)),
                 lambda: bc.prefix_weights(0, [pid] * 4, off, lens, q, lse, scores, [0] * 4),
                 lambda: bc.prefix_weights(0, [pid] * 2, [0, 900], [333, 77], q, lse, scores, [0] * 2),
                 lambda: bc.attend_window(0, [pid] * 4, [m] * 4, [5, 1999, 800, 0], off, lens, q, out, None, 4, 100, 0),
                 lambda: bc.project_prefix_layer(short, 0, h[:16], w_k, w_v)):
        best = 1e9
        for _ in range(12):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            start.record()
            call()
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        assert best < 1.0, best
    assert bc.device_status() == binding.OK

"""GPU parity of the rotary calls against the fp64 oracle.

Tolerance: the part of a turn enters as fp32 in [-1/8, 1/8) turn (2^-27 half turns, 2.4e-8 rad); cosine and sine are good
to 2 units in the last place (2^-23 below 1): they are off by at most E = 1.5e-7.  The factor and the products
and their sum are four fp32 roundings of 2^-24, each at most (|a| + |b|) scale.  One rounding to the type follows:
half a step, eps / 2 of the value."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from oracle import token_ops as op
from paper_2606_07571_b200 import binding, workloads

pytestmark = pytest.mark.gpu
E = 1.5e-7


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    binding.load_library()


def f64(t):
    return workloads.to_f64(t)


def make(hq, hkv, d, dtype):
    return binding.BiCache(1, hq, hkv, d, 8, dtype, 16, 1)


def rows_of(n, heads, d, dtype, seed, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((n, heads + pad, d), generator=g, device="cuda").to(dtype)
    return x[:, :heads]


def check(got, x, pos, freq, interleaved, scale, inverse, dtype):
    ref = op.rope(f64(x), pos, freq, interleaved, scale, inverse)
    pairs = len(freq)
    ax = np.abs(f64(x))
    d = np.arange(pairs)
    i, j = (2 * d, 2 * d + 1) if interleaved else (d, d + pairs)
    size = np.zeros_like(ax)
    size[..., i] = size[..., j] = ax[..., i] + ax[..., j]
    s = 1 / scale if inverse else scale
    inner = abs(s) * size * (E + 4 * 2.0 ** -24)
    err = np.abs(f64(got) - ref)
    assert (err <= inner + (np.abs(ref) + inner) * torch.finfo(dtype).eps / 2).all(), err.max()
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])      # dims beyond the rotated ones


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,rot", [(7, 1, 128, 128), (4, 4, 64, 64), (2, 1, 128, 32), (3, 3, 96, 20), (6, 2, 128, 2),
                                          (2, 2, 256, 256), (28, 4, 128, 108), (1, 1, 32, 16), (2, 2, 32, 30)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows(dtype, hq, hkv, d, rot, interleaved):
    bc = make(hq, hkv, d, dtype)
    n = 21
    q, k = rows_of(n, hq, d, dtype, 1, 1), rows_of(n, hkv, d, dtype, 2, 2)
    freq = binding.rope_frequencies(rot, 10000.0, "yarn", 4.0, 64, 1.0, 32.0)
    pos = torch.tensor([0, 1, 2, 5, 17, 100, 1000, 4095, 16384, 99999, 1 << 20, 3, 3, 3, 0, 7, -1, -1000, 65535, 12, 1],
                       dtype=torch.int32, device="cuda")
    p = pos.cpu().tolist()
    qo, ko = torch.full_like(rows_of(n, hq, d, dtype, 3, 1), 7), torch.empty_like(k)
    bc.rope(freq, q, qo, k, ko, positions=pos, interleaved=interleaved, attention_scale=1.25)
    check(qo, q, p, freq, interleaved, 1.25, False, dtype)
    check(ko, k, p, freq, interleaved, 1.25, False, dtype)
    q2 = q.clone()
    bc.rope(freq, q2, q2, positions=pos, interleaved=interleaved, attention_scale=1.25)       # in place, no keys
    assert torch.equal(q2, qo)
    back = torch.empty_like(k)
    bc.rope(freq, None, None, ko, back, positions=pos, interleaved=interleaved, attention_scale=1.25, inverse=True)
    check(back, ko, p, freq, interleaved, 1.25, True, dtype)
    # one in place, the other not: the dims beyond the rotated ones are still copied
    ko2 = torch.empty_like(k)
    q3 = q.clone()
    bc.rope(freq, q3, q3, k, ko2, positions=pos, interleaved=interleaved, attention_scale=1.25)
    assert torch.equal(q3, qo) and torch.equal(ko2, ko)


@pytest.mark.parametrize("rows", [0, 1, 2, 3, 5, 64, 1000, 2500])
def test_consecutive_positions_and_rows_behind_the_last(rows):
    bc = make(14, 2, 128, torch.bfloat16)
    freq = binding.rope_frequencies(128, 10000.0)
    q = rows_of(rows + 2, 14, 128, torch.bfloat16, 5)
    out = torch.full_like(q, 3)
    bc.rope(freq, q[:rows], out[:rows], position0=777)
    assert (out[rows:] == 3).all()
    check(out[:rows], q[:rows], range(777, 777 + rows), freq, False, 1.0, False, torch.bfloat16)


@pytest.mark.parametrize("rule,args", [("none", ()), ("linear", (4.0,)), ("ntk", (8.0,)), ("yarn", (16.0, 4096, 1.0, 32.0)),
                                       ("bands", (8.0, 8192, 1.0, 4.0))])
@pytest.mark.parametrize("rot", [2, 64, 128, 256])
def test_table(rule, args, rot):
    bc = make(2, 1, 128, torch.bfloat16)
    freq = binding.rope_frequencies(rot, 10000.0, rule, *args)
    pos = torch.tensor([0, 1, 3, 1000, (1 << 20) + 1, 2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")
    table = torch.empty((7, rot // 2, 2), device="cuda")
    bc.rope_table(freq, table, positions=pos, attention_scale=1.5)
    # the frequency itself is a double: 2^-53 of 2^31 radians is 2.4e-7 at the farthest position
    far = np.abs(np.array(pos.cpu().tolist(), dtype=np.float64))[:, None, None] * np.asarray(freq)[None, :, None] * 2.0 ** -52
    err = np.abs(f64(table) - op.rope_table(pos.cpu().tolist(), freq, 1.5))
    assert (err <= 1.5 * (E + 2 * 2.0 ** -24 + far)).all(), err.max()
    head = table.clone()
    bc.rope_table(freq, table, position0=5)
    np.testing.assert_allclose(f64(table), op.rope_table(range(5, 12), freq), atol=E + 2.0 ** -24)
    bc.rope_table(freq, head[:0], position0=5)


def test_far_rows_and_strides_past_32_bits():
    bc = make(1, 1, 128, torch.bfloat16)
    freq = binding.rope_frequencies(128, 10000.0)
    rows, stride = 600, 1 << 22                                   # the last rows start 2.5 G elements into the tensor
    big = torch.empty(stride * (rows - 1) + 128, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((rows, 1, 128), (stride, 128, 1))
    x.copy_(rows_of(rows, 1, 128, torch.bfloat16, 1))
    out = torch.empty((rows, 1, 128), dtype=torch.bfloat16, device="cuda")
    bc.rope(freq, None, None, x, out, position0=2 ** 31 - 700)    # positions run past 32 bits too
    ref = torch.empty_like(out)
    bc.rope(freq, None, None, x.contiguous(), ref, position0=2 ** 31 - 700)
    assert torch.equal(out, ref)
    near = torch.empty_like(out)
    pos = torch.arange(2 ** 31 - 700, 2 ** 31 - 100, device="cuda").to(torch.int32)
    bc.rope(freq, None, None, x.contiguous(), near, positions=pos)
    assert torch.equal(out, near)
    bc.rope(freq, None, None, x, x, position0=2 ** 31 - 700)
    assert torch.equal(x, ref)


def test_in_a_graph_and_on_another_stream():
    bc = make(4, 2, 128, torch.bfloat16)
    freq = binding.rope_frequencies(128, 10000.0)
    q, k = rows_of(50, 4, 128, torch.bfloat16, 1), rows_of(50, 2, 128, torch.bfloat16, 2)
    qo, ko, table = torch.empty_like(q), torch.empty_like(k), torch.empty((50, 64, 2), device="cuda")
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        bc.rope(freq, q, qo, k, ko, positions=pos)
        bc.rope_table(freq, table, positions=pos)
    freq[:] = 0                                                   # the call has taken its frequencies
    pos.add_(1000)                                                # positions are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    freq = binding.rope_frequencies(128, 10000.0)
    p = range(1000, 1050)
    check(qo, q, p, freq, False, 1.0, False, torch.bfloat16)
    check(ko, k, p, freq, False, 1.0, False, torch.bfloat16)
    np.testing.assert_allclose(f64(table), op.rope_table(p, freq), atol=E + 2.0 ** -24)


def test_rotated_queries_meet_keys_projected_with_the_table():
    """rope_table into project_prefix_layer, rope on queries and own keys, attend: the result does not change when
    all positions move by the same amount (up to the rounding of the rotated bf16 values)."""
    hq, hkv, d, m, n, d_model = 4, 2, 128, 96, 24, 256
    h, w_k, w_v = workloads.draw_hidden_and_weights(m, d_model, hkv, d, 3, device="cuda")
    freq = binding.rope_frequencies(d, 10000.0)
    q, k, v = (rows_of(n, x, d, torch.bfloat16, s) for x, s in ((hq, 1), (hkv, 2), (hkv, 3)))
    outs = []
    for shift in (0, 4096):
        bc = binding.BiCache(1, hq, hkv, d, 16, torch.bfloat16, 64, 2)
        pid, _, _ = bc.reserve_prefix(1, m)
        table = torch.empty((m, d // 2, 2), device="cuda")
        bc.rope_table(freq, table, position0=shift)
        bc.project_prefix_layer(pid, 0, h, w_k, w_v, rope=table)
        qr, kr, out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
        bc.rope(freq, q, qr, k, kr, position0=shift + m)
        bc.attend(0, [pid], [0], [n], qr, kr, v, out)
        assert bc.device_status() == 0
        outs.append(f64(out))
    # each side within the attention tests' 2e-2 of the exact result
    assert np.abs(outs[0] - outs[1]).max() <= 4e-2
    assert np.abs(outs[0]).max() > 0.1

"""CPU tests of the token-eviction and rotary calls: frequencies against the oracle, and every refusal the
host makes, through a host-only context (which answers UNSUPPORTED once the arguments are in order)."""
import ctypes as C

import numpy as np
import pytest

import __graft_entry__ as entry
from oracle import token_ops as op
from paper_2606_07571_b200 import binding as b

A16, A4, ODD = 0x10000, 0x10004, 0x10002          # pointers that are never followed


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return b.load_library()


@pytest.fixture
def ctx(lib):
    cfg = b.Config(3, 4, 2, 128, 16, 32, b.BF16, -1)
    c = C.c_void_p()
    assert lib.bicache_create(C.byref(cfg), C.byref(c)) == b.OK
    yield c
    lib.bicache_destroy(c)


def reserve(lib, ctx, key, m, first_layer=0):
    pid = C.c_int32(-1)
    assert lib.bicache_reserve_prefix_layers(ctx, C.c_uint64(key), m, first_layer, C.byref(pid), None, None, 0) == b.OK
    return pid.value


@pytest.mark.parametrize("rot", [2, 4, 44, 64, 128, 256])
@pytest.mark.parametrize("rule,factor,length,low,high", [
    ("none", 0.0, 0, 0, 0), ("linear", 4.0, 0, 0, 0), ("ntk", 8.0, 0, 0, 0), ("yarn", 16.0, 4096, 1.0, 32.0),
    ("yarn", 2.0, 1, 1.0, 32.0), ("bands", 8.0, 8192, 1.0, 4.0)])
def test_frequencies(lib, rot, rule, factor, length, low, high):
    for base in (10000.0, 500000.0):
        got = b.rope_frequencies(rot, base, rule, factor, length, low, high)
        # a handful of fp64 operations, one pow of up to 1 ulp, exponents up to 13 in the logarithm
        np.testing.assert_allclose(got, op.rope_frequencies(rot, base, rule, factor, length, low, high), rtol=1e-13)


@pytest.mark.parametrize("args", [
    (0, 1e4, "none", 1.0, 0, 1.0, 2.0), (3, 1e4, "none", 1.0, 0, 1.0, 2.0), (258, 1e4, "none", 1.0, 0, 1.0, 2.0),
    (64, 1.0, "none", 1.0, 0, 1.0, 2.0), (64, float("nan"), "none", 1.0, 0, 1.0, 2.0),
    (64, float("inf"), "none", 1.0, 0, 1.0, 2.0),
    (64, 1e4, "linear", 0.0, 0, 1.0, 2.0), (64, 1e4, "ntk", float("nan"), 0, 1.0, 2.0),
    (64, 1e4, "yarn", 2.0, 0, 1.0, 2.0), (64, 1e4, "yarn", 2.0, 4096, 0.0, 2.0), (64, 1e4, "bands", 2.0, 4096, 2.0, 2.0),
    (64, 1e4, "bands", 2.0, 4096, 1.0, float("inf")), (64, 1e4, "unheard of", 2.0, 4096, 1.0, 2.0)])
def test_frequency_refusals(lib, args):
    with pytest.raises(b.BiCacheError) as ei:
        b.rope_frequencies(*args)
    assert ei.value.status == b.ERR_INVALID


def weights(lib, ctx, layer=0, pid=(0,), off=(0,), n=(4,), q=A16, qs=512, lse=A4, sin=None, sout=A4, so=(0,), hs=64,
            decay=0.0, scale=0.1, R=None):
    i32, i64 = (lambda a: None if a is None else (C.c_int32 * max(len(a), 1))(*a)), \
               (lambda a: None if a is None else (C.c_int64 * max(len(a), 1))(*a))
    return lib.bicache_prefix_weights(ctx, layer, len(pid or ()) if R is None else R, i32(pid), i64(off), i32(n), q, qs,
                                      lse, sin, sout, i64(so), hs, decay, scale, None)


def test_weights_refusals(lib, ctx):
    p0, p1, late = reserve(lib, ctx, 1, 40), reserve(lib, ctx, 2, 64), reserve(lib, ctx, 3, 16, first_layer=1)
    ok = dict(pid=(p0,))
    assert weights(lib, ctx, **ok) == b.ERR_UNSUPPORTED                        # in order; no device path here
    assert weights(lib, ctx, pid=(-1, p0, p0, p1), off=(0,) * 4, n=(1, 2, 0, 3), so=(-9, 0, 0, 128)) == b.ERR_UNSUPPORTED
    assert weights(lib, ctx, pid=(late,), layer=1) == b.ERR_UNSUPPORTED
    assert weights(lib, ctx, pid=(), off=(), n=(), so=(), q=None, lse=None, sout=None) == b.ERR_UNSUPPORTED
    for bad in (dict(layer=-1), dict(layer=3), dict(R=-1), dict(off=None), dict(n=None), dict(so=None), dict(q=None),
                dict(lse=None), dict(sout=None), dict(q=A4), dict(lse=ODD), dict(sout=ODD), dict(sin=ODD),
                dict(qs=511), dict(qs=516), dict(n=(-1,)), dict(off=(-1,)), dict(so=(-1,)), dict(hs=39),
                dict(decay=0.5), dict(decay=float("nan"), sin=A4), dict(scale=float("inf"))):
        assert weights(lib, ctx, **dict(ok, **bad)) == b.ERR_INVALID, bad
    two = dict(off=(0, 4), n=(4, 4))
    assert weights(lib, ctx, pid=(p0, p0), so=(0, 1), **two) == b.ERR_INVALID              # one prefix, two blocks
    assert weights(lib, ctx, pid=(p0, p1), so=(0, 64 + 39), **two) == b.ERR_INVALID        # blocks overlap
    assert weights(lib, ctx, pid=(p0, p1), so=(0, 64 + 40), **two) == b.ERR_UNSUPPORTED
    assert weights(lib, ctx, pid=(p0, p1, p0), off=(0,) * 3, n=(1,) * 3, so=(0, 200, 400)) == b.ERR_INVALID
    assert weights(lib, ctx, pid=(late,)) == b.ERR_INVALID                                 # owns nothing in layer 0
    assert weights(lib, ctx, pid=(-2,)) == b.ERR_INVALID
    assert weights(lib, ctx, pid=(99,)) == b.ERR_NOTFOUND
    assert weights(lib, None) == b.ERR_INVALID


def test_select_refusals(lib, ctx):
    def call(rows=2, n=10, scores=A4, ss=10, keep=4, first=1, last=1, idx=A4, xs=4, c=ctx):
        return lib.bicache_select_tokens(c, rows, n, scores, ss, keep, first, last, idx, xs, None)
    assert call() == b.ERR_UNSUPPORTED
    assert call(rows=1, ss=0, xs=0) == b.ERR_UNSUPPORTED                       # strides of a single row are not read
    assert call(keep=10, first=50, last=50, xs=10) == b.ERR_UNSUPPORTED        # protected ends cut to the row
    assert call(rows=0, scores=None, idx=None) == b.ERR_UNSUPPORTED
    for bad in (dict(rows=-1), dict(rows=2 ** 31), dict(n=-1), dict(n=2 ** 30 + 1, ss=2 ** 31, keep=4), dict(keep=-1), dict(keep=11), dict(first=-1), dict(last=-1),
                dict(first=3, last=2), dict(keep=9, first=50, last=50), dict(scores=None), dict(idx=None),
                dict(scores=ODD), dict(idx=ODD), dict(ss=9), dict(xs=3), dict(c=None)):
        assert call(**bad) == b.ERR_INVALID, bad


def test_compact_refusals(lib, ctx):
    src, dst, late = reserve(lib, ctx, 1, 40), reserve(lib, ctx, 2, 20), reserve(lib, ctx, 3, 20, first_layer=2)

    def call(s=src, d=dst, l0=0, nl=3, keep=20, idx=A4, ls=20, hs=0, c=ctx):
        return lib.bicache_compact_prefix(c, s, d, l0, nl, keep, idx, ls, hs, None)
    assert call() == b.ERR_UNSUPPORTED
    assert call(d=late, l0=2, nl=1) == b.ERR_UNSUPPORTED
    for bad in (dict(d=src, keep=40), dict(l0=-1), dict(l0=1), dict(nl=-1), dict(nl=4), dict(l0=2 ** 31 - 1, nl=1), dict(d=late),
                dict(keep=19), dict(idx=None), dict(idx=ODD), dict(ls=-1), dict(hs=-1), dict(c=None)):
        assert call(**bad) == b.ERR_INVALID, bad
    assert call(s=77) == b.ERR_NOTFOUND and call(d=77) == b.ERR_NOTFOUND


def test_rope_refusals(lib, ctx):
    def call(rows=3, pos=A4, rot=128, f=(0.5,) * 64, scale=1.0, q=A16, qs=512, qo=A16, qos=512, k=A16, ks=256, ko=A16 * 2,
             kos=264, c=ctx):
        f = None if f is None else (C.c_double * len(f))(*f)
        return lib.bicache_rope(c, rows, pos, 0, rot, 0, 0, f, scale, q, qs, qo, qos, k, ks, ko, kos, None)
    assert call() == b.ERR_UNSUPPORTED
    assert call(k=None, ko=None, pos=None) == b.ERR_UNSUPPORTED
    assert call(q=None, qo=None, rows=0) == b.ERR_UNSUPPORTED
    for bad in (dict(rows=-1), dict(rot=0), dict(rot=7), dict(rot=130), dict(f=None), dict(f=(float("inf"),) * 64), dict(f=(-2.0 ** 21,) * 64),
                dict(scale=0.0), dict(scale=float("nan")), dict(pos=ODD), dict(q=None), dict(qo=None), dict(k=None),
                dict(q=None, qo=None, k=None, ko=None), dict(q=A4), dict(ko=A4), dict(qs=504), dict(kos=255),
                dict(qs=516), dict(qs=520), dict(c=None)):
        assert call(**bad) == b.ERR_INVALID, bad

    def table(rows=3, pos=None, rot=64, f=(0.5,) * 32, scale=1.0, t=A16, c=ctx):
        f = None if f is None else (C.c_double * len(f))(*f)
        return lib.bicache_rope_table(c, rows, pos, 0, rot, f, scale, t, None)
    assert table() == b.ERR_UNSUPPORTED and table(rows=0) == b.ERR_UNSUPPORTED
    for bad in (dict(rows=-1), dict(rot=0), dict(rot=9), dict(rot=258), dict(f=None), dict(f=(float("nan"),) * 32),
                dict(scale=0.0), dict(t=None), dict(t=A4), dict(pos=ODD), dict(c=None)):
        assert table(**bad) == b.ERR_INVALID, bad


def test_rope_refuses_one_output_for_both_tensors_and_an_infinite_inverse_scale(lib, ctx):
    f = (C.c_double * 64)(*[0.5] * 64)

    def call(inverse=0, scale=1.0, qo=A16, ko=A16 * 2, rows=3):
        return lib.bicache_rope(ctx, rows, None, 0, 128, 0, inverse, f, scale, A16 * 3, 512, qo, 512, A16 * 4, 256, ko, 512, None)
    assert call() == b.ERR_UNSUPPORTED
    assert call(ko=A16) == b.ERR_INVALID
    assert call(ko=A16, rows=0) == b.ERR_UNSUPPORTED             # no rows: the address is not used
    # 2^-140: a subnormal whose reciprocal is not finite
    assert call(scale=2.0 ** -140) == b.ERR_UNSUPPORTED
    assert call(inverse=1, scale=2.0 ** -140) == b.ERR_INVALID

"""CPU tests of the calls on a growing cache: every refusal that the host makes, through a host-only context (which answers
UNSUPPORTED once the arguments are in order)."""
import ctypes as C

import numpy as np
import pytest

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding as b

A16, B16, C16, A4, ODD = 0x10000, 0x20000, 0x30000, 0x10004, 0x10002      # pointers that are never followed
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return b.load_library()


@pytest.fixture
def ctx(lib):
    cfg = b.Config(3, 4, 2, 128, 16, 32, b.BF16, -1)          # rows of 512 and 256 elements
    c = C.c_void_p()
    assert lib.bicache_create(C.byref(cfg), C.byref(c)) == b.OK
    for key, m, first in ((1, 40, 0), (2, 17, 1), (3, 16, 0)):
        pid = C.c_int32(-1)
        assert lib.bicache_reserve_prefix_layers(c, C.c_uint64(key), m, first, C.byref(pid), None, None, 0) == b.OK
        assert pid.value == key - 1
    yield c
    lib.bicache_destroy(c)


def host(a, dtype):
    return None if a is None else np.array(a, dtype=dtype)


def at(a):
    return None if a is None else a.ctypes.data


def rotation(pairs=64, axes=1, scale=1.0, freq=None, axis=None, interleaved=0, rot_dim=None, null_freq=False):
    f = np.ones(max(pairs, 1)) if freq is None else np.array(freq, dtype=np.float64)
    x = None if axis is None else np.array(axis, dtype=np.int32)
    s = b.RotationStruct(2 * pairs if rot_dim is None else rot_dim, interleaved, axes, scale, None if null_freq else at(f), at(x))
    s.keep = (f, x)
    return s


def append(lib, ctx, layer=0, pid=(0, 2), tok=(30, 0), off=(0, 10), n=(10, 16), k=A16, v=B16, ks=256, q=None, qs=512,
           qo=None, qos=512, rot="plain", pos=None, axis_stride=0, R=None):
    args = host(pid, np.int32), host(tok, np.int32), host(off, np.int64), host(n, np.int32)
    r = rotation() if rot == "plain" else rot
    return lib.bicache_append_tokens(ctx, layer, len(pid) if R is None else R, *map(at, args), k, v, ks, q, qs, qo, qos,
                                     None if r is None else C.addressof(r), pos, axis_stride, None)


@pytest.mark.parametrize("change", [
    {}, {"q": C16, "qo": C16}, {"q": C16, "qo": 0x40000, "qs": 1024}, {"rot": None}, {"pos": A4}, {"n": (0, 0), "k": None, "v": None},
    {"pid": (), "tok": (), "off": (), "n": ()}, {"tok": (0, 0), "n": (40, 16)}, {"pid": (0, 0), "tok": (30, 20), "n": (10, 10)},
    {"pid": (0, 0), "tok": (30, 30), "n": (10, 0)}, {"layer": 2, "pid": (1, 2), "tok": (7, 0)}, {"ks": 264}, {"off": (0, 0)},
    {"rot": rotation(axes=3, axis=[0, 1, 2, 0] * 16), "pos": A16, "axis_stride": 26}, {"rot": rotation(pairs=1)}])
def test_append_arguments_in_order(lib, ctx, change):
    assert append(lib, ctx, **change) == b.ERR_UNSUPPORTED


@pytest.mark.parametrize("change", [
    {"layer": -1}, {"layer": 3}, {"R": -1}, {"pid": None, "R": 2}, {"tok": None}, {"off": None}, {"n": None}, {"n": (-1, 1)},
    {"off": (-1, 0)}, {"tok": (-1, 0)}, {"tok": (31, 0)}, {"tok": (0x7fffffff, 0)}, {"n": (0x7fffffff, 1)}, {"tok": (41, 0), "n": (0, 1)},
    {"pid": (1, 2), "tok": (0, 0), "n": (4, 4)},              # layer 0 of a prefix that owns layers 1 and 2
    {"pid": (0, 0), "tok": (30, 29), "n": (10, 2)}, {"pid": (0, 2, 0), "tok": (5, 0, 5), "off": (0, 1, 2), "n": (1, 1, 1)},
    {"k": None}, {"v": None}, {"k": A4}, {"v": ODD}, {"ks": 255}, {"ks": 260},
    {"q": C16}, {"qo": C16}, {"q": C16, "qo": C16, "rot": None}, {"q": A4, "qo": C16}, {"q": C16, "qo": ODD},
    {"q": C16, "qo": 0x40000, "qs": 511}, {"q": C16, "qo": 0x40000, "qos": 516}, {"q": C16, "qo": C16, "qs": 1024},
    {"q": C16, "qo": A16}, {"q": C16, "qo": B16}, {"pos": ODD},
    {"rot": rotation(axes=0)}, {"rot": rotation(axes=5), "pos": A16, "axis_stride": 99}, {"rot": rotation(pairs=65)},
    {"rot": rotation(rot_dim=0)}, {"rot": rotation(rot_dim=63)}, {"rot": rotation(null_freq=True)}, {"rot": rotation(scale=0.0)},
    {"rot": rotation(scale=INF)}, {"rot": rotation(pairs=2, freq=[1.0, NAN])}, {"rot": rotation(pairs=2, freq=[1.0, 2.0 ** 21])},
    {"rot": rotation(axes=2, axis=[0, 2] * 32), "pos": A16, "axis_stride": 26}, {"rot": rotation(axis=[1] + [0] * 63)},
    {"rot": rotation(axes=2, axis=[0, -1] * 32), "pos": A16, "axis_stride": 26},
    {"rot": rotation(axes=2), "axis_stride": 26}, {"rot": rotation(axes=2), "pos": A16, "axis_stride": 25},
    {"off": (0, 9), "q": C16, "qo": 0x40000}])
def test_append_refusals(lib, ctx, change):
    assert append(lib, ctx, **change) == b.ERR_INVALID


def test_append_unknown_prefix(lib, ctx):
    assert append(lib, ctx, pid=(0, 7)) == b.ERR_NOTFOUND
    assert append(lib, ctx, pid=(0, -1)) == b.ERR_NOTFOUND
    assert append(lib, None) == b.ERR_INVALID


def read(lib, ctx, layer=0, pid=(0, 0), tok=(30, 30), off=(0, 10), n=(10, 10), k=A16, v=B16, ks=256):
    args = host(pid, np.int32), host(tok, np.int32), host(off, np.int64), host(n, np.int32)
    return lib.bicache_read_tokens(ctx, layer, len(pid), *map(at, args), k, v, ks, None)


def test_read(lib, ctx):
    assert read(lib, ctx) == b.ERR_UNSUPPORTED                # the same token twice may be read
    for change in ({"layer": 3}, {"n": (11, 1)}, {"n": (-1, 1)}, {"k": None}, {"v": A4}, {"k": A16, "v": A16}, {"ks": 248},
                   {"ks": 257}, {"pid": (1, 1), "tok": (0, 0)}, {"tok": None}, {"off": (0, 9)}):
        assert read(lib, ctx, **change) == b.ERR_INVALID
    assert read(lib, ctx, pid=(0, 9)) == b.ERR_NOTFOUND


def window(lib, ctx, layer=0, pid=(0, 2, 0), cached=(40, 3, 0), pos=(30, 0, 7), off=(0, 10, 20), n=(10, 3, 2), q=A16,
           qs=512, out=B16, os=512, lse=None, sinks=0, left=-1, right=-1, scale=0.1, R=None):
    args = host(pid, np.int32), host(cached, np.int32), host(pos, np.int32), host(off, np.int64), host(n, np.int32)
    return lib.bicache_attend_window(ctx, layer, len(pid) if R is None else R, *map(at, args), q, qs, out, os, lse, sinks, left,
                                     right, scale, None)


BIG = 0x7fffffff


@pytest.mark.parametrize("change", [
    {}, {"lse": A4}, {"sinks": BIG, "left": BIG, "right": BIG}, {"left": 0, "right": 0}, {"scale": 0.0}, {"scale": -1.0},
    {"pid": (-1, 2, 0), "cached": (0, 3, 0)}, {"pos": (BIG - 10, 0, 0)}, {"n": (0, 0, 0), "q": None, "out": None},
    {"pid": (), "cached": (), "pos": (), "off": (), "n": ()}, {"layer": 1, "pid": (1, 2, 0), "cached": (17, 0, 0)}, {"qs": 640, "os": 768}])
def test_window_arguments_in_order(lib, ctx, change):
    assert window(lib, ctx, **change) == b.ERR_UNSUPPORTED


@pytest.mark.parametrize("change", [
    {"layer": -1}, {"layer": 3}, {"R": -1}, {"pid": None, "R": 3}, {"cached": None}, {"pos": None}, {"off": None}, {"n": None},
    {"sinks": -1}, {"left": -2}, {"right": -2}, {"scale": NAN}, {"scale": INF}, {"n": (-1, 0, 0)}, {"off": (0, -1, 0)},
    {"pos": (0, 0, -1)}, {"cached": (-1, 0, 0)}, {"cached": (41, 0, 0)}, {"pos": (BIG - 9, 0, 0)}, {"pid": (-2, 2, 0)},
    {"pid": (-1, 2, 0)}, {"pid": (1, 2, 0), "cached": (1, 0, 0)}, {"q": None}, {"out": None}, {"q": A4}, {"out": ODD},
    {"lse": ODD}, {"out": A16}, {"qs": 504}, {"os": 508}, {"qs": 516}, {"n": (0x60000000, 3, 2)}, {"off": (0, 11, 10)}])
def test_window_refusals(lib, ctx, change):
    assert window(lib, ctx, **change) == b.ERR_INVALID


def test_window_unknown_prefix(lib, ctx):
    assert window(lib, ctx, pid=(0, 2, 5)) == b.ERR_NOTFOUND
    assert window(lib, None) == b.ERR_INVALID


def axes(lib, ctx, rows=5, rot="plain", pos=A4, stride=5, inverse=0, q=A16, qs=512, qo=B16, qos=512, k=None, ks=0, ko=None, kos=0):
    r = rotation(axes=3, axis=[0, 1, 2, 0] * 16) if rot == "plain" else rot
    return lib.bicache_rope_axes(ctx, rows, None if r is None else C.addressof(r), pos, stride, inverse, q, qs, qo, qos, k, ks,
                                 ko, kos, None)


def test_axes(lib, ctx):
    for change in ({}, {"inverse": 1}, {"rows": 0, "pos": None, "q": None, "qo": None}, {"qo": A16},
                   {"k": C16, "ko": C16, "ks": 256, "kos": 256}, {"rot": rotation(), "stride": 0}):
        assert axes(lib, ctx, **change) == b.ERR_UNSUPPORTED
    for change in ({"rows": -1}, {"rot": None}, {"pos": None}, {"pos": ODD}, {"stride": 4}, {"q": None}, {"qo": None}, {"q": A4},
                   {"qs": 511}, {"qos": 520 - 4}, {"qo": A16, "qs": 1024}, {"k": C16, "ko": B16, "ks": 256, "kos": 256},
                   {"rot": rotation(pairs=65)}, {"rot": rotation(axes=5)}, {"rot": rotation(axis=[0] * 63 + [1])},
                   {"rot": rotation(scale=1e-42), "inverse": 1}):
        assert axes(lib, ctx, **change) == b.ERR_INVALID
    assert axes(lib, None) == b.ERR_INVALID


def test_axes_table(lib, ctx):
    def table(rows=5, rot="plain", pos=A4, stride=5, out=A16, c=ctx):
        r = rotation(pairs=128, axes=4, axis=[0, 1, 2, 3] * 32) if rot == "plain" else rot
        return lib.bicache_rope_axes_table(c, rows, None if r is None else C.addressof(r), pos, stride, out, None)
    assert table() == table(rows=0, pos=None, out=None) == b.ERR_UNSUPPORTED
    for change in ({"rows": -1}, {"rot": None}, {"pos": None}, {"out": None}, {"out": A4}, {"stride": 4}, {"c": None},
                   {"rot": rotation(pairs=129)}):
        assert table(**change) == b.ERR_INVALID


def test_rotation_object():
    r = b.Rotation([1.0, 0.5], interleaved=True, attention_scale=2.0, pair_axis=[0, 1], num_axes=2)
    assert (r.struct.rot_dim, r.struct.interleaved, r.struct.num_axes, r.struct.attention_scale) == (4, 1, 2, 2.0)
    with pytest.raises(AssertionError):
        b.Rotation([1.0, 0.5], pair_axis=[0], num_axes=2)

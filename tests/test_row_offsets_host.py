"""CPU tests of row offsets whose last row has no 64-bit number: refused by every call that takes a ragged batch, not taken for
a batch without rows."""
import ctypes as C

import numpy as np
import pytest

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding as b

A, B, C16, A4 = 0x10000, 0x20000, 0x30000, 0x10004             # pointers that are never followed
END = 2 ** 63 - 1


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return b.load_library()


@pytest.fixture
def ctx(lib):
    cfg = b.Config(1, 4, 2, 128, 16, 32, b.BF16, -1)
    c = C.c_void_p()
    assert lib.bicache_create(C.byref(cfg), C.byref(c)) == b.OK
    pid = C.c_int32(-1)
    assert lib.bicache_reserve_prefix(c, C.c_uint64(1), 40, C.byref(pid), None, None, 0) == b.OK
    assert pid.value == 0
    yield c
    lib.bicache_destroy(c)


def i32(*x):
    return np.array(x, dtype=np.int32)


def calls(lib, ctx, off, n):
    """Name and answer of every call for the batch of the request given and one of three rows."""
    pid, off, n = i32(0, 0), np.array([off, 0], dtype=np.int64), i32(n, 3)
    tok, zero, cached = i32(0, 37), i32(0, 0), i32(40, 40)
    p = [x.ctypes.data for x in (pid, off, n, tok, zero, cached)]
    pid_, off_, n_, tok_, zero_, cached_ = p
    score = np.zeros(2, dtype=np.int64)
    # an answer of UNSUPPORTED: the arguments are in order, and the context has no device
    yield "append", lib.bicache_append_tokens(ctx, 0, 2, pid_, tok_, off_, n_, A, B, 256, None, 0, None, 0, None, None, 0, None)
    yield "read", lib.bicache_read_tokens(ctx, 0, 2, pid_, tok_, off_, n_, A, B, 256, None)
    yield "window", lib.bicache_attend_window(ctx, 0, 2, pid_, cached_, zero_, off_, n_, A, 512, B, 512, None, 0, -1, -1,
                                              C.c_float(0.1), None)
    yield "weights", lib.bicache_prefix_weights(ctx, 0, 2, pid_, off_, n_, A, 512, A4, None, A4, score.ctypes.data, 40, 0.0, 0.1, None)


@pytest.mark.parametrize("off,n", [(END, 1), (END - 9, 10), (END, 30)])
def test_the_last_row_has_no_number(lib, ctx, off, n):
    assert dict(calls(lib, ctx, off, n)) == {name: b.ERR_INVALID for name in ("append", "read", "window", "weights")}


@pytest.mark.parametrize("off,n", [(END - 10, 10), (END, 0), (3, 10)])
def test_the_last_row_has_one(lib, ctx, off, n):
    assert dict(calls(lib, ctx, off, n)) == {name: b.ERR_UNSUPPORTED for name in ("append", "read", "window", "weights")}


def test_calls_that_choose_per_request(lib, ctx):
    """bicache_attend_layer and bicache_attend_step: a request that reuses its prefix starts behind it."""
    def layer(off, n, depth):
        a = [np.array(x, dtype=t) for x, t in (([depth], np.int32), ([0], np.int32), ([off], np.int64), ([n], np.int32))]
        return lib.bicache_attend_layer(ctx, 0, 1, *(C.cast(x.ctypes.data, C.POINTER(C.c_int32 if x.dtype == np.int32 else C.c_int64))
                                                     for x in a), A, B, C16, 512, 256, 0x40000, 512, None, C.c_float(0.1), None)

    def step(off, n, depth):
        a = [np.array(x, dtype=t) for x, t in (([depth], np.int32), ([0], np.int32), ([-1], np.int32), ([off], np.int64), ([n], np.int32))]
        return lib.bicache_attend_step(ctx, 0, 1, 4, 1, *(C.cast(x.ctypes.data, C.POINTER(C.c_int32 if x.dtype == np.int32 else C.c_int64))
                                                          for x in a), A, B, C16, 512, 256, 0x40000, 512, None, C.c_float(0.1), None)
    for depth in (0, 1):                                       # not reused, reused
        for call in (layer, step):
            assert call(END - 40, 41, depth) == b.ERR_INVALID
            assert call(END - 41, 41, depth) == b.ERR_UNSUPPORTED

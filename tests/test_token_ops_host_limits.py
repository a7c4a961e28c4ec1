"""CPU tests of the token-eviction and rotary calls at the ends of their arguments' ranges, through a host-only context
(which answers UNSUPPORTED once the arguments are in order)."""
import ctypes as C

import numpy as np
import pytest

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding as b

A16, A4 = 0x10000, 0x10004                        # pointers that are never followed


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


def test_positions_beyond_what_the_angles_hold_are_refused(lib, ctx):
    f = (C.c_double * 64)(*[0.5] * 64)

    def rope(position0, rows=3, pos=None):
        return lib.bicache_rope(ctx, rows, pos, position0, 128, 0, 0, f, 1.0, A16, 512, A16, 512, None, 0, None, 0, None)

    def table(position0, rows=3, pos=None):
        return lib.bicache_rope_table(ctx, rows, pos, position0, 128, f, 1.0, A16, None)
    for call in (rope, table):
        for position0 in (-2 ** 36, -5, 0, 2 ** 31, 2 ** 36 - 2):
            assert call(position0) == b.ERR_UNSUPPORTED, position0
        for position0 in (-2 ** 63, -2 ** 36 - 1, 2 ** 36 - 1, 2 ** 50, 2 ** 63 - 1):
            assert call(position0) == b.ERR_INVALID, position0
            assert call(position0, pos=A4) == b.ERR_UNSUPPORTED        # the positions are an array: not read
            assert call(position0, rows=0) == b.ERR_UNSUPPORTED
        assert call(0, rows=2 ** 36 + 2) == b.ERR_INVALID


@pytest.mark.parametrize("args", [
    (4, 1e4, "ntk", 1e-300, 0, 1.0, 2.0),         # the base becomes 0
    (128, 1e4, "linear", 5e-324, 0, 1.0, 2.0), (128, 1e4, "yarn", 5e-324, 4096, 1.0, 32.0),
    (128, 1e4, "bands", 5e-324, 8192, 1.0, 4.0)])
def test_factors_that_leave_no_finite_frequency_are_refused(lib, args):
    with pytest.raises(b.BiCacheError) as ei:
        b.rope_frequencies(*args)
    assert ei.value.status == b.ERR_INVALID


def test_far_scaling_that_stays_finite_is_not_refused(lib):
    for args in ((4, 1e4, "ntk", 1e300, 0, 1.0, 2.0), (128, 1e4, "linear", 1e300, 0, 1.0, 2.0),
                 (128, 1e4, "linear", 1e-300, 0, 1.0, 2.0)):
        assert np.isfinite(b.rope_frequencies(*args)).all()


def test_compaction_of_no_layers_needs_no_list(lib, ctx):
    ids = []
    for key, m in ((1, 40), (2, 20)):
        pid = C.c_int32(-1)
        assert lib.bicache_reserve_prefix_layers(ctx, C.c_uint64(key), m, 0, C.byref(pid), None, None, 0) == b.OK
        ids.append(pid.value)

    def call(num_layers, idx, keep=20):
        return lib.bicache_compact_prefix(ctx, *ids, 1, num_layers, keep, idx, 20, 0, None)
    assert call(0, None) == b.ERR_UNSUPPORTED     # an empty tensor has no address
    assert call(0, A4) == b.ERR_UNSUPPORTED
    assert call(1, None) == b.ERR_INVALID and call(0, None, keep=19) == b.ERR_INVALID

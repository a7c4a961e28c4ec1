"""CPU tests of how the binding packs a call's host arrays: values that do not fit are refused, whatever holds them."""
import struct

import numpy as np
import pytest

from paper_2606_07571_b200 import binding as b


@pytest.mark.parametrize("code,values", [("i", [0, -1, 5, 2 ** 31 - 1, -2 ** 31]), ("q", [0, -1, 2 ** 40, 2 ** 63 - 1])])
def test_values_that_fit(code, values):
    want = struct.pack("%d%s" % (len(values), code), *values)
    for a in (values, tuple(values), np.array(values, dtype=np.int64), np.array(values * 2, dtype=np.int64)[:len(values)],
              np.array(values, dtype=np.int64)[::-1][::-1], np.array(values, dtype=object)):
        assert b._host_list(a, code) == (want, len(values))
    small = np.array([3, 0, 7], dtype=np.uint8)
    assert b._host_list(small, code)[0] == struct.pack("3" + code, 3, 0, 7)
    assert b._host_list([], code) == (b"", 0) and b._host_list(np.empty(0), code) == (b"", 0)


@pytest.mark.parametrize("value", [2 ** 31, -2 ** 31 - 1, 2 ** 32 + 5, 2 ** 40])
@pytest.mark.parametrize("count", [1, 100])
def test_values_that_do_not_fit(value, count):
    values = [1] * (count - 1) + [value]
    for a in (values, np.array(values, dtype=np.int64)):
        with pytest.raises((struct.error, OverflowError)):
            b._host_list(a, "i")


def test_fractions():
    for a in ([1.5], np.array([1.5])):
        with pytest.raises((struct.error, OverflowError)):
            b._host_list(a, "i")


@pytest.mark.parametrize("count", [1, 8, 9, 100])              # by a loop, by arrays
@pytest.mark.parametrize("dtype", [np.int32, np.int64, list])
def test_rows_past_the_tensor(count, dtype):
    def within(off, n, rows):
        off, n = [0] * (count - 1) + [off], [5] * (count - 1) + [n]
        if dtype is not list:
            off, n = np.array(off, dtype=dtype), np.array(n, dtype=dtype)
        return b._rows_within(off, n, b._host_list(off, "q")[0], b._host_list(n, "i")[0], rows)
    assert within(20, 10, 30) and not within(21, 10, 30) and not within(20, 11, 30)
    assert not within(2 ** 31 - 5, 10, 30) and not within(2 ** 31 - 1, 2 ** 31 - 1, 30)
    assert not within(2 ** 31 - 5, 10, 2 ** 31) and within(2 ** 31 - 5, 10, 2 ** 31 + 5)


def test_rows_in_lists_of_numpy_numbers():
    off, n = [np.int32(2 ** 31 - 5), np.int32(0)], [np.int32(10), np.int32(0)]
    assert not b._rows_within(off, n, b._host_list(off, "q")[0], b._host_list(n, "i")[0], 30)
    none = np.empty(0, dtype=np.int32)
    assert b._rows_within(none, none, b"", b"", 0)

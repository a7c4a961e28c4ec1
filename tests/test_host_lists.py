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

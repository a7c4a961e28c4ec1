"""CPU tests of the binding's look at the rows of a batch: a request without rows has none, wherever it says that they begin."""
import pytest

from paper_2606_07571_b200 import binding as b


@pytest.mark.parametrize("count", [3, 40])                     # by a loop; by arrays
@pytest.mark.parametrize("empty_at,rows,within", [(0, 30, True), (10 ** 6, 30, True), (2 ** 40, 30, True), (0, 29, False)])
def test_rows_of_empty_requests(count, empty_at, rows, within):
    off, n = [0, 10, 20] + [empty_at] * (count - 3), [10, 10, 10] + [0] * (count - 3)
    off[1], n[1] = empty_at, 0
    packed_off, _ = b._host_list(off, "q")
    packed_n, _ = b._host_list(n, "i")
    assert b._rows_within(off, n, packed_off, packed_n, rows) == within


@pytest.mark.parametrize("count", [3, 40])
def test_no_rows_at_all(count):
    off, n = [7] * count, [0] * count
    assert b._rows_within(off, n, b._host_list(off, "q")[0], b._host_list(n, "i")[0], 0)

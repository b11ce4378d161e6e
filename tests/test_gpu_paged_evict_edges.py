"""Eviction where weights are -infinity and pages do not exist."""

import pytest

from test_gpu_paged import torch_cuda  # noqa: F401
from test_gpu_paged_evict import Evictable

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,capacity", [(500, 500), (9000, 9000), (500, 20000), (18000, 20000)])
def test_rows_without_a_page_go_in_front_of_weights_of_minus_infinity(torch_cuda, rows, capacity):  # noqa: F811
    # a row without a page has less weight than any number, the least one included: it stays only where all others do
    torch = torch_cuda
    gone = [1, 4, 5, 17]                                        # pages; the table's other ones exist
    missing = {r for i in gone for r in range(16 * i, 16 * i + 16)}
    there = [r for r in range(rows) if r not in missing]
    for keep, last, most in ((len(there) // 2, 0, 0), (len(there), 3, 0), (len(there) + 10, 1, 0), (40, 8, 7)):
        c = Evictable(torch, rows, [rows], keep, capacity=capacity, heads=2, group=1, D=8).randomise()
        c.weights.fill_(float("-inf"))
        for r in there[20: 20 + most]:                          # and a few that are numbers
            c.weights[0, int(c.table[0, r // 16]), :, r % 16] = -float(r)
        for n, i in enumerate(gone):
            c.table[0, i] = (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31)[n]
        c.evict(0, last)
        forced = list(range(rows - last, rows))
        rest = there[20: 20 + most] + [r for r in there if r not in there[20: 20 + most]] + sorted(missing)
        want = sorted(forced + [r for r in rest if r not in set(forced)][: keep - last])
        assert c.rows_out.tolist() == [want, want], (keep, last)

"""The eviction's largest calls (no GPU needed)."""

import pytest

from test_host_logic import lib  # noqa: F401
from test_paged_evict_host import _call
from test_paged_host import _pages

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("page,max_pages,keep,status", [
    (16, 2 ** 26, 2 ** 28, 2), (16, 2 ** 26, 2 ** 28 - 15, 2), (16, 2 ** 26, 2 ** 28 - 16, 3), (16, 2 ** 26, MOST, 2), (16, 2 ** 24, MOST, 2), (16, 2 ** 24 - 1, MOST, 3),
    (64, 2 ** 24, 2 ** 30, 2), (64, 2 ** 24, 2 ** 30 - 64, 3), (128, 2 ** 23, MOST, 3), (256, 2 ** 22, MOST, 3), (16, 10, MOST, 3)], ids=str)
def test_more_pages_than_a_grid_has_workgroups_are_refused(lib, page, max_pages, keep, status):  # noqa: F811
    # 2^24 workgroups of 256 threads would be 2^32; what is not refused for that is, here, for its workspace
    pages = _pages(page_size=page, max_pages=max_pages, k_stride=dict(enumerate([80 * page * 64, 2 * page * 64, page * 64, 64])),
                   v_stride=dict(enumerate([80 * page * 64, 2 * page * 64, page * 64, 64])))
    assert _call(lib, pages, keep=keep, ws=None) == status
    assert ("2^24" in lib.sablock_last_error().decode()) == (status == 2)

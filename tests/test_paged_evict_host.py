"""Refusals of the eviction, by the library and by its Python call (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import lib  # noqa: F401
from test_paged_binding import H, I32, MOST, N, NL, PAGE, PAGES, Called, _tensors, no_gpu  # noqa: F401
from test_paged_host import BAD_PAGES, FAKE, _pages


def _call(lib, pages=None, **changed):  # noqa: F811
    a = dict(table=FAKE, lengths=FAKE, keep=40, first=4, last=8, after=2 * FAKE, len_out=3 * FAKE, rows_out=FAKE, weights=FAKE, kp=FAKE, vp=FAKE, bounds=None,
             ws=FAKE, ws_bytes=1 << 40)
    a.update(changed)
    return lib.sablock_evict_paged(ctypes.byref(pages or _pages()), *a.values(), None)


@pytest.mark.parametrize("change,status", BAD_PAGES, ids=[str(c[0]) for c in BAD_PAGES])
def test_caches(lib, change, status):  # noqa: F811
    assert _call(lib, _pages(**change)) == status
    n = ctypes.c_size_t(7)
    assert lib.sablock_evict_paged_workspace_bytes(ctypes.byref(_pages(**change)), ctypes.byref(n)) == status and n.value == 7


def test_arguments(lib):  # noqa: F811
    for name in ("table", "lengths", "after", "len_out", "rows_out", "weights", "kp", "vp"):
        assert _call(lib, **{name: None}) == 1, name
        assert lib.sablock_last_error().decode().startswith("sablock_evict_paged"), name
    for name in ("weights", "kp", "vp", "bounds", "ws"):
        assert _call(lib, **{name: FAKE + 8}) == 1, name
    assert _call(lib, after=FAKE) == 1 and _call(lib, len_out=FAKE) == 1
    assert _call(lib, ws=None) == 3 and _call(lib, ws_bytes=64) == 3
    for bad in (dict(keep=0, first=0, last=0), dict(keep=-1), dict(first=-1), dict(last=-1), dict(first=33), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
        assert _call(lib, **bad) == 1, bad


def test_workspace(lib):  # noqa: F811
    n = ctypes.c_size_t(0)
    assert lib.sablock_evict_paged_workspace_bytes(ctypes.byref(_pages()), ctypes.byref(n)) == 0
    assert n.value >= 3 * 2 * 2 * 160 * 4                       # a key for every row that the table has room for
    assert lib.sablock_evict_paged_workspace_bytes(None, ctypes.byref(n)) == 1 and lib.sablock_evict_paged_workspace_bytes(ctypes.byref(_pages()), None) == 1


def _evict(t, **changed):
    a = dict(weights=torch.zeros((NL, PAGES, H, PAGE)), after=torch.zeros((N, MOST), dtype=I32), len_out=torch.zeros(N, dtype=I32),
             rows_out=torch.zeros((N * NL * H, 30), dtype=I32))
    a.update(changed)
    B.sablock_evict_paged(t["pages"], t["table"], t["lengths"], a["weights"], t["k_pool"], t["v_pool"], 30, a["after"], a["len_out"], a["rows_out"], t["ws"],
                          bounds=t["bounds"])


def test_binding(no_gpu):  # noqa: F811
    with pytest.raises(Called):
        _evict(_tensors())
    for name, bad in (("weights", torch.zeros((NL, PAGES, H, PAGE), dtype=torch.bfloat16)), ("weights", torch.zeros((NL, PAGES - 1, H, PAGE))),
                      ("weights", torch.zeros((NL, H, PAGES, PAGE)).transpose(1, 2)), ("len_out", torch.zeros(N - 1, dtype=I32)),
                      ("rows_out", torch.zeros((N * NL * H, 29), dtype=I32)), ("rows_out", torch.zeros((N * NL * H, 30))), ("after", torch.zeros((N, MOST - 1), dtype=I32))):
        with pytest.raises(ValueError, match="dense"):
            _evict(_tensors(), **{name: bad})
    with pytest.raises(ValueError, match="page table of 7 entries"):
        _evict(_tensors(), after=torch.zeros((N, MOST + 1), dtype=I32))
    for name, match in (("k_pool", "^K pool"), ("v_pool", "^V pool"), ("bounds", "dense"), ("lengths", "dense")):
        t = _tensors()
        t[name] = t[name][:-1].clone()
        with pytest.raises(ValueError, match=match):
            _evict(t)

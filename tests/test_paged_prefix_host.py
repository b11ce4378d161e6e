"""Refusals of the attention with common prefixes, by the library and by its Python call (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import lib  # noqa: F401
from test_paged_binding import I32, MOST, N, Called, _tensors, no_gpu  # noqa: F401
from test_paged_host import BAD_PAGES, FAKE, _pages


def _call(lib, pages=None, **changed):  # noqa: F811
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, lengths=FAKE, begin=FAKE, n_pages=FAKE, n=2, out=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(changed)
    return lib.sablock_decode_prefix_paged(ctypes.byref(pages or _pages()), *a.values(), None)


@pytest.mark.parametrize("change,status", BAD_PAGES + [(dict(n_q_heads=34), 2), (dict(head_dim=48), 2), (dict(head_dim=24, dtype=0), 2), (dict(n_seq=4, max_pages=1 << 26), 2)], ids=lambda c: str(c))
def test_caches(lib, change, status):  # noqa: F811
    assert _call(lib, _pages(**change)) == status
    n = ctypes.c_size_t(7)
    assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(_pages(**change)), 1, ctypes.byref(n)) == status and n.value == 7


def test_arguments(lib):  # noqa: F811
    for name in ("q", "kp", "vp", "table", "lengths", "begin", "n_pages", "out"):
        assert _call(lib, **{name: None}) == 1, name
        assert lib.sablock_last_error().decode().startswith("sablock_decode_prefix_paged"), name
    for name in ("q", "kp", "vp", "ws"):
        assert _call(lib, **{name: FAKE + 8}) == 1, name
    assert _call(lib, ws=None) == 3 and _call(lib, ws_bytes=64) == 3
    for n, status in ((0, 1), (-1, 1), (4097, 2)):
        assert _call(lib, n=n) == status
        size = ctypes.c_size_t(7)
        assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(_pages()), n, ctypes.byref(size)) == status and size.value == 7


def test_workspace(lib):  # noqa: F811
    size, plain = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.sablock_decode_paged_workspace_bytes(ctypes.byref(_pages()), ctypes.byref(plain)) == 0
    for n in (1, 5, 4096):
        assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(_pages()), n, ctypes.byref(size)) == 0 and size.value > plain.value
    assert lib.sablock_decode_prefix_paged_workspace_bytes(None, 1, ctypes.byref(size)) == 1
    # 12 problems of 2^26 steps and one are 805 306 380, below 2^30; 16 of them, above, are refused
    assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(_pages(n_seq=3, max_pages=1 << 26)), 1, ctypes.byref(size)) == 0
    assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(_pages()), 1, None) == 1


def _decode(t, begin=None, pages=None):
    begin, pages = torch.zeros(3, dtype=I32) if begin is None else begin, torch.zeros(2, dtype=I32) if pages is None else pages
    B.sablock_decode_prefix_paged(t["pages"], t["q_out"], t["k_pool"], t["v_pool"], t["table"], t["lengths"], begin, pages, t["out"], t["ws"])


def test_binding(no_gpu):  # noqa: F811
    with pytest.raises(Called):
        _decode(_tensors())
    for begin in (torch.zeros(2, dtype=I32), torch.zeros(3), torch.zeros((3, 2), dtype=I32)[:, 0]):
        with pytest.raises(ValueError, match="dense"):
            _decode(_tensors(), begin)
    with pytest.raises(ValueError, match="dense"):
        _decode(_tensors(), pages=torch.zeros(2, dtype=torch.int64))
    for name, match in (("k_pool", "^K pool"), ("v_pool", "^V pool"), ("q_out", "dense"), ("out", "dense"), ("lengths", "dense")):
        t = _tensors()
        t[name] = t[name][:-1].clone()
        with pytest.raises(ValueError, match=match):
            _decode(t)
    t = _tensors()
    t["table"] = torch.zeros((N, MOST + 1), dtype=I32)
    with pytest.raises(ValueError, match="page table of 7 entries"):
        _decode(t)

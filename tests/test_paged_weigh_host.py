"""Refusals of the attention that gathers weights, by the library and by its Python call (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import lib  # noqa: F401
from test_paged_binding import H, I32, MOST, N, NL, PAGE, PAGES, Called, _tensors, no_gpu  # noqa: F401
from test_paged_host import BAD_PAGES, FAKE, _pages

NAN = float("nan")


def _call(lib, pages=None, **changed):  # noqa: F811
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, lengths=FAKE, n_new=1, counts=None, decay=1.0, weights=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(changed)
    return lib.sablock_decode_weighed_paged(ctypes.byref(pages or _pages()), *a.values(), None)


@pytest.mark.parametrize("change,status", BAD_PAGES + [(dict(n_q_heads=34), 2), (dict(head_dim=48), 2), (dict(head_dim=24, dtype=0), 2)], ids=lambda c: str(c))
def test_caches(lib, change, status):  # noqa: F811
    assert _call(lib, _pages(**change)) == status
    n = ctypes.c_size_t(7)
    assert lib.sablock_decode_weighed_paged_workspace_bytes(ctypes.byref(_pages(**change)), ctypes.byref(n)) == status and n.value == 7


def test_arguments(lib):  # noqa: F811
    for name in ("q", "kp", "vp", "table", "lengths", "weights", "out"):
        assert _call(lib, **{name: None}) == 1, name
        assert lib.sablock_last_error().decode().startswith("sablock_decode_weighed_paged"), name
    for name in ("q", "kp", "vp", "weights", "ws"):
        assert _call(lib, **{name: FAKE + 8}) == 1, name
    assert _call(lib, ws=None) == 3 and _call(lib, ws_bytes=64) == 3
    for bad in (dict(n_new=-1), dict(decay=-0.5), dict(decay=NAN), dict(decay=float("inf"))):
        assert _call(lib, **bad) == 1, bad


def test_workspace(lib):  # noqa: F811
    n, plain = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.sablock_decode_weighed_paged_workspace_bytes(ctypes.byref(_pages()), ctypes.byref(n)) == 0
    assert lib.sablock_decode_paged_workspace_bytes(ctypes.byref(_pages()), ctypes.byref(plain)) == 0
    assert n.value >= plain.value + 3 * 2 * 8 * 160 * 4         # a logit for every row that the table has room for, and query head
    assert lib.sablock_decode_weighed_paged_workspace_bytes(None, ctypes.byref(n)) == 1
    assert lib.sablock_decode_weighed_paged_workspace_bytes(ctypes.byref(_pages()), None) == 1


def _decode(t, weights=None, counts=None):
    weights = torch.zeros((NL, PAGES, H, PAGE)) if weights is None else weights
    B.sablock_decode_weighed_paged(t["pages"], t["q_out"], t["k_pool"], t["v_pool"], t["table"], t["lengths"], weights, t["out"], t["ws"], counts=counts)


def test_binding(no_gpu):  # noqa: F811
    with pytest.raises(Called):
        _decode(_tensors(), counts=torch.zeros(N, dtype=I32))
    for bad in (torch.zeros((NL, PAGES, H, PAGE), dtype=torch.bfloat16), torch.zeros((NL, PAGES - 1, H, PAGE)), torch.zeros((NL, H, PAGES, PAGE)).transpose(1, 2)):
        with pytest.raises(ValueError, match="dense"):
            _decode(_tensors(), weights=bad)
    for bad in (torch.zeros(N - 1, dtype=I32), torch.zeros(N)):
        with pytest.raises(ValueError, match="dense"):
            _decode(_tensors(), counts=bad)
    for name, match in (("k_pool", "^K pool"), ("v_pool", "^V pool"), ("q_out", "dense"), ("out", "dense"), ("lengths", "dense")):
        t = _tensors()
        t[name] = t[name][:-1].clone()
        with pytest.raises(ValueError, match=match):
            _decode(t)
    t = _tensors()
    t["table"] = torch.zeros((N, MOST + 1), dtype=I32)
    with pytest.raises(ValueError, match="page table of 7 entries"):
        _decode(t)

"""Refusals of the append with norms, by the library and by its Python call (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import lib  # noqa: F401
from test_paged_binding import D, G, H, N, NL, Called, _tensors, no_gpu  # noqa: F401
from test_paged_host import BAD_PAGES, FAKE, _pages, _tokens

NAN = float("nan")


def _call(lib, pages=None, tokens=None, norms=None, **changed):  # noqa: F811
    a = dict(q=FAKE, k=FAKE, v=FAKE, qw=FAKE, kw=FAKE, counts=None, pos=FAKE, freq=FAKE, table=FAKE, lengths=FAKE, q_out=2 * FAKE, kp=FAKE, vp=FAKE, bounds=FAKE)
    a.update(changed)
    norms = B.make_head_norms() if norms is None else norms
    return lib.sablock_append_normed_paged(ctypes.byref(pages or _pages()), ctypes.byref(tokens or _tokens()), ctypes.byref(norms), *a.values(), None)


def test_layout_of_the_norms():
    assert ctypes.sizeof(B.CHeadNorms) == 16 and B.CHeadNorms.per_head.offset == 4
    n = B.make_head_norms(1e-5, per_head=True)
    assert n.eps == ctypes.c_float(1e-5).value and n.per_head == 1


@pytest.mark.parametrize("change,status", BAD_PAGES, ids=[str(c[0]) for c in BAD_PAGES])
def test_caches(lib, change, status):  # noqa: F811
    assert _call(lib, _pages(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(n_new=0), 1), (dict(n_new=161), 1), (dict(rotary_dim=80), 1), (dict(rotary_dim=24), 2), (dict(interleaved=2), 1), (dict(reserved=1), 1),
    (dict(k_stride={0: -8}), 1), (dict(q_stride={1: 12}), 2), (dict(k_stride={3: 56}), 1)], ids=str)
def test_new_tokens(lib, change, status):  # noqa: F811
    assert _call(lib, tokens=_tokens(**change)) == status


def test_arguments(lib):  # noqa: F811
    for name in ("q", "k", "v", "qw", "kw", "table", "lengths", "q_out", "kp", "vp", "pos", "freq"):
        assert _call(lib, **{name: None}) == 1, name
        assert lib.sablock_last_error().decode().startswith("sablock_append_normed_paged"), name
    for name in ("q", "k", "v", "qw", "kw", "q_out", "kp", "vp", "bounds"):
        assert _call(lib, **{name: FAKE + 8}) == 1, name
    assert _call(lib, q_out=FAKE) == 1
    assert lib.sablock_append_normed_paged(ctypes.byref(_pages()), ctypes.byref(_tokens()), None, *[FAKE] * 10, 2 * FAKE, *[FAKE] * 3, None) == 1


@pytest.mark.parametrize("norms", [B.CHeadNorms(0.0, 0), B.CHeadNorms(-1e-6, 0), B.CHeadNorms(NAN, 0), B.CHeadNorms(float("inf"), 0), B.CHeadNorms(1e-6, 2),
                                   B.CHeadNorms(1e-6, -1), B.CHeadNorms(1e-6, 0, (ctypes.c_int32 * 2)(0, 1))], ids=lambda n: f"{n.eps}-{n.per_head}-{n.reserved[1]}")
def test_norms(lib, norms):  # noqa: F811
    assert _call(lib, norms=norms) == 1


def _append(t, per_head=False, **changed):
    w = {"q_weight": torch.ones((NL, H * G, D) if per_head else (NL, D)), "k_weight": torch.ones((NL, H, D) if per_head else (NL, D))}
    w.update(changed)
    B.sablock_append_normed_paged(t["pages"], t["tokens"], B.make_head_norms(1e-6, per_head), t["k"], t["v"], t["positions"], t["freq"], t["table"], t["lengths"],
                                  t["k_pool"], t["v_pool"], q=t["q"], q_out=t["q_out"], bounds=t["bounds"], **w)


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("n_new", [1, 5])
def test_binding(no_gpu, n_new, per_head):  # noqa: F811
    with pytest.raises(Called):
        _append(_tensors(n_new), per_head)
    with pytest.raises(Called):                                 # without queries their weight is not looked for
        t = _tensors(n_new)
        t["q"] = t["q_out"] = None
        _append(t, per_head, q_weight=None)
    heads = H * G if per_head else 1
    for bad in (torch.ones((NL, heads, D), dtype=torch.bfloat16), torch.ones(NL * heads * D - 1), torch.ones((NL, heads, 2 * D))[..., ::2]):
        with pytest.raises(ValueError, match="dense"):
            _append(_tensors(n_new), per_head, q_weight=bad)
    with pytest.raises(ValueError, match="dense"):
        _append(_tensors(n_new), per_head, k_weight=torch.ones(NL * (H if per_head else 1) * D - 4))
    for what, match in (("k", "^k: "), ("q", "^q: "), ("v", "^v: "), ("k_pool", "^K pool: "), ("lengths", "dense")):
        t = _tensors(n_new)
        t[what] = t[what][:-1].clone()
        with pytest.raises(ValueError, match=match):
            _append(t, per_head)
    assert N == 3

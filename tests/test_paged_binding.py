"""The paged cache's Python calls refuse tensors that their descriptors do not describe, before the library is asked (no GPU needed)."""

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import lib  # noqa: F401

BF, I32 = torch.bfloat16, torch.int32
N, NL, H, G, D, PAGE, PAGES, MOST = 3, 2, 2, 4, 64, 16, 20, 6


class Called(Exception):
    pass


@pytest.fixture
def no_gpu(lib, monkeypatch):  # noqa: F811
    """Host tensors count as the current device's, and every call of the library raises."""
    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise Called(name)
            return call

    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda *a: None)
    library = Library()
    monkeypatch.setattr(B, "load", lambda: library)


def _tensors(n_new=1):
    pool = lambda: torch.zeros((NL, PAGES, H, PAGE, D), dtype=BF)  # noqa: E731
    qkv = torch.zeros((N, n_new, NL, H * (G + 2), D), dtype=BF).permute(0, 2, 3, 1, 4)
    t = dict(k_pool=pool(), v_pool=pool(), table=torch.zeros((N, MOST), dtype=I32), lengths=torch.zeros(N, dtype=I32), positions=torch.zeros(N, dtype=I32),
             q=qkv[:, :, : H * G], k=qkv[:, :, H * G: H * (G + 1)], v=qkv[:, :, H * (G + 1):], freq=torch.zeros(D // 2),
             q_out=torch.zeros((N, NL, H * G, n_new, D), dtype=BF), bounds=torch.zeros((NL, PAGES, H, 2, D), dtype=BF), ws=torch.zeros(1 << 16, dtype=torch.uint8),
             out=torch.zeros((N, NL, H * G, D)), idx=torch.zeros((N * NL * H, 30), dtype=I32), kv=torch.zeros((N, NL, H, 70, D), dtype=BF),
             list=torch.zeros((N * NL * H, 4), dtype=I32))
    t["pages"] = B.make_pages(t["k_pool"], t["v_pool"], t["table"], H * G)
    t["tokens"] = B.make_new_tokens(t["k"], t["v"], t["q"])
    t["shape"] = B.make_shape(torch.zeros((N, NL, H * G, 8, D), dtype=BF), t["kv"])
    return t


def _append(t):
    B.sablock_append_paged(t["pages"], t["tokens"], t["k"], t["v"], t["positions"], t["freq"], t["table"], t["lengths"], t["k_pool"], t["v_pool"], q=t["q"],
                           q_out=t["q_out"], bounds=t["bounds"])


def _decode(t):
    B.sablock_decode_paged(t["pages"], t["q_out"], t["k_pool"], t["v_pool"], t["table"], t["lengths"], t["out"], t["ws"])


def _select(t):
    B.sablock_select_pages(t["pages"], t["q_out"], t["bounds"], t["table"], t["lengths"], 4, t["list"], t["ws"])


def _compact(t):
    B.sablock_compact_paged(t["shape"], t["kv"], t["kv"], t["idx"], 30, True, t["pages"], t["table"], t["k_pool"], t["v_pool"], bounds=t["bounds"], lengths_out=t["lengths"])


CALLS = {"append": _append, "decode": _decode, "select": _select, "compact": _compact}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("n_new", [1, 5])
def test_tensors_of_the_descriptor_reach_the_library(no_gpu, name, n_new):
    with pytest.raises(Called):
        CALLS[name](_tensors(n_new))


def _fewer(axis):
    return lambda x: x.narrow(axis, 0, x.shape[axis] - 1)


STRIDED = [("of fewer sequences", _fewer(0)), ("of fewer layers", _fewer(1)), ("of fewer heads", _fewer(2)), ("dense", lambda x: x.contiguous()),
           ("of another type", lambda x: x.float()), ("of other axes, too short", lambda x: x[-1, -1, -1]), ("heads repeated", lambda x: x[:, :, :1].expand_as(x)),
           ("copied in another order", lambda x: x.transpose(1, 2).contiguous().transpose(1, 2))]


@pytest.mark.parametrize("n_new", [1, 5])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("change", [c[1] for c in STRIDED], ids=[c[0] for c in STRIDED])
def test_append_refuses_new_tokens_that_the_descriptor_does_not_describe(no_gpu, what, change, n_new):
    t = _tensors(n_new)
    t[what] = change(t[what])
    with pytest.raises(ValueError, match=f"^{what}: the descriptor says"):
        _append(t)


def test_append_refuses_queries_that_its_descriptor_was_made_without(no_gpu):
    # their strides would be zero: every sequence's and head's query would be the first one
    t = _tensors()
    t["tokens"] = B.make_new_tokens(t["k"], t["v"])
    with pytest.raises(ValueError, match="^q: the descriptor says"):
        _append(t)
    t["q"] = t["q_out"] = None
    with pytest.raises(Called):
        _append(t)


@pytest.mark.parametrize("name", ["append", "decode", "compact"])
@pytest.mark.parametrize("what", ["k_pool", "v_pool"])
@pytest.mark.parametrize("change", [("fewer layers", _fewer(0)), ("fewer pages", lambda x: x[:, :-1].contiguous()), ("smaller pages", _fewer(3)), ("another type", lambda x: x.float()),
                                    ("another order", lambda x: x.transpose(2, 3).contiguous().transpose(2, 3)), ("flat, too short", lambda x: x.flatten()[1:])], ids=lambda c: c[0])
def test_pools_that_the_descriptor_does_not_describe(no_gpu, name, what, change):
    t = _tensors()
    t[what] = change[1](t[what])
    with pytest.raises(ValueError, match="^%s pool: the descriptor says" % what[0].upper()):
        CALLS[name](t)


@pytest.mark.parametrize("name", CALLS)
def test_tables_of_another_width(no_gpu, name):
    t = _tensors()
    t["table"] = torch.zeros((N, MOST + 1), dtype=I32)
    with pytest.raises(ValueError, match="page table of 7 entries"):
        CALLS[name](t)
    t["table"] = torch.zeros((N, MOST - 1), dtype=I32)
    with pytest.raises(ValueError, match="dense"):
        CALLS[name](t)


def test_tensors_that_hold_more_than_the_descriptor_says(no_gpu):
    # a batch's buffers with room for more sequences, layers and pages; axes with one entry, whose strides say nothing; other axes over the same memory
    t = _tensors(5)
    big = torch.zeros((N + 2, 5, NL, H * (G + 2), D), dtype=BF).permute(0, 2, 3, 1, 4)
    t["q"], t["k"], t["v"] = big[:, :, : H * G], big[:, :, H * G: H * (G + 1)], big[:, :, H * (G + 1):]
    t["k_pool"] = torch.zeros((NL + 1, PAGES, H, PAGE, D), dtype=BF)
    t["v_pool"] = t["v_pool"].flatten()
    for name in CALLS:
        with pytest.raises(Called):
            CALLS[name](t)
    one = torch.zeros((1, 1, H * G, 1, D), dtype=BF)
    assert B._extent("k", one.shape, (7, 0, D, 3, 1)).dense == H * G * D           # strides of single entries
    B._strided(BF, (one, B._extent("k", one.shape, (7, 0, D, 3, 1))), (one.expand(4, 2, -1, -1, -1), B._extent("k", (4, 2, H * G, 1, D), (0, 0, D, 9, 1))))
    wide = torch.zeros((3, 4 * D), dtype=BF)
    B._strided(BF, (wide, B._extent("k", (3, 1, 2, 1, D), (4 * D, 0, 2 * D, 0, 1))))
    for short in (wide[:2], wide.flatten()[D + 1:]):            # the last element looked at is 11 D - 1
        with pytest.raises(ValueError, match="^k: "):
            B._strided(BF, (short.contiguous().clone(), B._extent("k", (3, 1, 2, 1, D), (4 * D, 0, 2 * D, 0, 1))))

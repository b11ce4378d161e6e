"""The paged cache's calls on the host: layouts, refusals, and what the kernels make of table entries and lengths (no GPU needed)."""

import ctypes
import os
import re

import pytest
import torch

from paper_2510_22556_amd import binding as B
from test_host_logic import ROOT, _run_host_code, _shape, lib  # noqa: F401

FAKE = 0x1000                                  # never followed: refusals come first


def _pages(**kw):
    c = B.CPages()
    c.n_seq, c.n_layers, c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype = 3, 2, 8, 2, 64, B.SABLOCK_BF16
    c.page_size, c.n_pages, c.max_pages, c.compute_units = 16, 40, 10, 256
    for a, x in enumerate([40 * 2 * 16 * 64, 2 * 16 * 64, 16 * 64, 64]):
        c.k_stride[a] = c.v_stride[a] = x
    for k, v in kw.items():
        if isinstance(v, dict):
            for a, x in v.items():
                getattr(c, k)[a] = x
        else:
            setattr(c, k, v)
    return c


def _tokens(**kw):
    t = B.CNewTokens()
    t.n_new, t.rotary_dim = 4, 64
    for s, h in ((t.q_stride, 8), (t.k_stride, 2), (t.v_stride, 2)):
        for a, x in enumerate([2 * h * 4 * 64, h * 4 * 64, 4 * 64, 64]):
            s[a] = x
    for k, v in kw.items():
        if isinstance(v, dict):
            for a, x in v.items():
                getattr(t, k)[a] = x
        else:
            setattr(t, k, v)
    return t


def test_layouts_match_the_header():
    hdr = open(os.path.join(ROOT, "include", "sablock.h")).read()
    for struct, name in ((B.CPages, "sablock_pages"), (B.CNewTokens, "sablock_new_tokens")):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, hdr).group(1)
        assert re.findall(r"int(?:32|64)_t\s+(\w+)", body) == [f[0] for f in struct._fields_]
    assert ctypes.sizeof(B.CPages) == 12 * 4 + 8 * 8 and B.CPages.k_stride.offset == 48
    assert ctypes.sizeof(B.CNewTokens) == 4 * 4 + 12 * 8 and B.CNewTokens.q_stride.offset == 16


BAD_PAGES = [
    (dict(n_seq=0), 1), (dict(n_layers=0), 1), (dict(n_kv_heads=0), 1), (dict(n_q_heads=3), 1), (dict(dtype=2), 1), (dict(dtype=-1), 1),
    (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(page_size=0), 1), (dict(compute_units=-1), 1), (dict(reserved={0: 1}), 1),
    (dict(reserved={1: 1}), 1), (dict(k_stride={1: -8}), 1), (dict(v_stride={3: 56}), 1), (dict(k_stride={2: 0}), 1), (dict(v_stride={0: 0}), 1),
    (dict(head_dim=12), 2), (dict(head_dim=264), 2), (dict(head_dim=0), 2), (dict(page_size=8), 2), (dict(page_size=24), 2),
    (dict(page_size=512), 2), (dict(n_seq=4097, n_layers=1), 2), (dict(n_seq=4000, n_layers=9), 2), (dict(max_pages=(1 << 26) + 1), 2),
    (dict(k_stride={3: 68}), 2), (dict(v_stride={1: 2 * 16 * 64 + 4}), 2)]


def _calls(lib, pages, tokens, **null):  # noqa: F811
    """Status of every call for one cache; names in `null` become NULL, other values replace arguments."""
    a = dict(q=FAKE, k=FAKE, v=FAKE, idx=FAKE, table=FAKE, lengths=FAKE, kp=FAKE, vp=FAKE, bounds=FAKE, q_out=2 * FAKE, counts=None, positions=FAKE,
             freq=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40, plist=None, n_listed=0, n_pick=4, n_first=1, n_last=1, list_out=FAKE, budget=96)
    a.update(null)
    pg, tk = ctypes.byref(pages), ctypes.byref(tokens)
    shape = _shape(n_seq=pages.n_seq, n_layers=pages.n_layers, n_kv_heads=2, n_q_heads=8, head_dim=64, dtype=B.SABLOCK_BF16)
    return {
        "compact": lambda: lib.sablock_compact_paged(ctypes.byref(shape), a["k"], a["v"], a["idx"], a["budget"], 1, pg, a["table"], a["kp"], a["vp"],
                                                     a["bounds"], None, None),
        "append": lambda: lib.sablock_append_paged(pg, tk, a["q"], a["k"], a["v"], a["counts"], a["positions"], a["freq"], a["table"], a["lengths"],
                                                   a["q_out"], a["kp"], a["vp"], a["bounds"], None),
        "decode": lambda: lib.sablock_decode_paged(pg, a["q"], a["kp"], a["vp"], a["table"], a["lengths"], a["plist"], a["n_listed"], a["out"], a["ws"],
                                                   a["ws_bytes"], None),
        "select": lambda: lib.sablock_select_pages(pg, a["q"], a["bounds"], a["table"], a["lengths"], a["n_pick"], a["n_first"], a["n_last"],
                                                   a["list_out"], a["ws"], a["ws_bytes"], None),
    }


@pytest.mark.parametrize("change,status", BAD_PAGES, ids=[str(c[0]) for c in BAD_PAGES])
def test_caches_that_no_call_takes(lib, change, status):  # noqa: F811
    pages = _pages(**change)
    for name, call in _calls(lib, pages, _tokens()).items():
        if name == "compact" and (pages.n_seq < 1 or pages.n_seq > 64 or pages.n_layers < 1):
            continue                           # its shape is refused first
        assert call() == status, name
        assert lib.sablock_last_error().decode().startswith("sablock_"), name
    n = ctypes.c_size_t(7)
    for f in (lib.sablock_decode_paged_workspace_bytes, lib.sablock_select_pages_workspace_bytes):
        assert f(ctypes.byref(pages), ctypes.byref(n)) == status and n.value == 7
        assert f(None, ctypes.byref(n)) == 1 and f(ctypes.byref(_pages()), None) == 1


def test_strides_of_axes_with_one_entry_are_not_looked_at(lib):  # noqa: F811
    n = ctypes.c_size_t(0)
    one = _pages(n_layers=1, n_kv_heads=1, n_q_heads=4, n_pages=1, k_stride={0: -1, 1: 3, 2: 5}, v_stride={0: 1, 1: -7, 2: 0})
    assert lib.sablock_decode_paged_workspace_bytes(ctypes.byref(one), ctypes.byref(n)) == 0 and n.value > 0


def test_null_and_misaligned_arguments(lib):  # noqa: F811
    ok = _pages()
    wrong = {"compact": ["k", "v", "idx", "table", "kp", "vp"], "append": ["k", "v", "table", "lengths", "kp", "vp", "q", "q_out", "positions", "freq"],
             "decode": ["q", "kp", "vp", "table", "lengths", "out"], "select": ["q", "bounds", "table", "lengths", "list_out"]}
    for call, names in wrong.items():
        for name in names:
            assert _calls(lib, ok, _tokens(), **{name: None})[call]() == 1, (call, name)
    odd = {"compact": ["k", "v", "kp", "vp", "bounds"], "append": ["q", "k", "v", "q_out", "kp", "vp", "bounds"], "decode": ["q", "kp", "vp", "ws"],
           "select": ["q", "bounds", "ws"]}
    for call, names in odd.items():
        for name in names:
            assert _calls(lib, ok, _tokens(), **{name: FAKE + 8})[call]() == 1, (call, name)
    for call in ("decode", "select"):
        assert _calls(lib, ok, _tokens(), ws=None)[call]() == 3
        assert _calls(lib, ok, _tokens(), ws_bytes=16)[call]() == 3


def test_refusals_of_compact(lib):  # noqa: F811
    assert _calls(lib, _pages(), _tokens(), budget=-1)["compact"]() == 1
    assert _calls(lib, _pages(), _tokens(), budget=145)["compact"]() == 1          # 145 + 16 rows, 160 have a place
    for change in (dict(n_kv_heads=4, k_stride={2: 16 * 64}), dict(head_dim=32), dict(dtype=0)):
        pages = _pages(**change)
        shape = _shape(n_seq=3, n_layers=2, n_kv_heads=2, n_q_heads=8, head_dim=64, dtype=1)
        args = (ctypes.byref(shape), FAKE, FAKE, FAKE, 96, 1, ctypes.byref(pages), FAKE, FAKE, FAKE, FAKE, None, None)
        assert lib.sablock_compact_paged(*args) == 1


@pytest.mark.parametrize("change,status", [
    (dict(n_new=0), 1), (dict(n_new=161), 1), (dict(rotary_dim=-16), 1), (dict(rotary_dim=80), 1), (dict(rotary_dim=24), 2), (dict(interleaved=2), 1),
    (dict(reserved=1), 1), (dict(k_stride={0: -8}), 1), (dict(v_stride={2: 100}), 2), (dict(q_stride={1: 12}), 2), (dict(k_stride={3: 56}), 1),
    (dict(q_stride={3: 0}), 1)], ids=str)
def test_refusals_of_append(lib, change, status):  # noqa: F811
    assert _calls(lib, _pages(), _tokens(**change))["append"]() == status


def test_append_refuses_its_own_input_as_output(lib):  # noqa: F811
    assert _calls(lib, _pages(), _tokens(), q_out=FAKE)["append"]() == 1


def test_refusals_of_decode_and_select(lib):  # noqa: F811
    def both(**kw):
        c = _calls(lib, _pages(**kw), _tokens())
        return c["decode"](), c["select"]()

    assert both(n_q_heads=34) == (2, 2)                         # 17 heads per KV head
    assert both(head_dim=56)[0] == 2 and both(head_dim=48)[0] == 2
    assert _calls(lib, _pages(head_dim=24, dtype=0), _tokens())["decode"]() == 2
    assert _calls(lib, _pages(), _tokens(), plist=FAKE, n_listed=0)["decode"]() == 1
    for bad in (dict(n_pick=0, n_first=0, n_last=0), dict(n_first=-1), dict(n_last=-1), dict(n_first=3, n_last=2), dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1)):
        assert _calls(lib, _pages(), _tokens(), **bad)["select"]() == 1


def test_entries_and_lengths_that_name_nothing(tmp_path):
    # what every kernel asks before it follows an entry of the table or takes a length
    rows = _run_host_code(tmp_path, """
#include "sablock_internal.h"
#include <climits>
#include <cstdio>
int main()
{
    sablock::PageDims d{};
    d.n_pages = 40; d.max_pages = 3; d.page = 16; d.shift = 4;
    const int32_t table[6] = {0, 39, 40, -1, INT_MAX, INT_MIN}, len[6] = {0, -1, INT_MIN, 47, 48, INT_MAX};
    for (int i = 0; i < 6; ++i) std::printf("%d %d\\n", sablock::page_at(d, table, i / 3, i % 3), sablock::rows_of(d, len, i));
}
""")
    assert rows == [[0, 0], [39, 0], [-1, 0], [-1, 47], [-1, 48], [-1, 48]]


def test_descriptors_from_tensors():
    k = torch.zeros((2, 40, 4, 16, 64), dtype=torch.bfloat16)
    v = torch.zeros((40, 2, 16, 4, 64), dtype=torch.bfloat16).permute(1, 0, 3, 2, 4)       # another order of the axes
    c = B.make_pages(k, v, torch.zeros((3, 7), dtype=torch.int32), 12)
    assert (c.n_seq, c.n_layers, c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype, c.page_size, c.n_pages, c.max_pages) == (3, 2, 12, 4, 64, 1, 16, 40, 7)
    assert list(c.k_stride) == [40 * 4 * 16 * 64, 4 * 16 * 64, 16 * 64, 64] and list(c.v_stride) == [4 * 16 * 64, 2 * 4 * 16 * 64, 64, 4 * 64]
    qkv = torch.zeros((3, 5, 2, 20, 64)).permute(0, 2, 3, 1, 4)
    t = B.make_new_tokens(qkv[:, :, 12:16], qkv[:, :, 16:], qkv[:, :, :12], interleaved=True)
    assert (t.n_new, t.rotary_dim, t.interleaved) == (5, 64, 1) and list(t.q_stride) == [5 * 2 * 20 * 64, 20 * 64, 64, 2 * 20 * 64]


def test_binding_refuses_tensors_that_the_kernels_could_not_follow(lib):  # noqa: F811
    i32 = dict(dtype=torch.int32)
    for bad in (torch.zeros(3), torch.zeros(3, dtype=torch.int64), torch.zeros(2, **i32), torch.zeros((3, 2), **i32)[:, 0], torch.zeros((2, 3), **i32).t()):
        with pytest.raises(ValueError, match="dense"):
            B._dense(torch.int32, 3, None, bad)
    B._dense(torch.int32, 3, None, torch.zeros(3, **i32), torch.zeros((2, 3), **i32))
    pages, k = _pages(), torch.zeros((1, 1, 2, 1, 64), dtype=torch.bfloat16)
    for call in (lambda: B.sablock_append_paged(pages, _tokens(), k, k, None, None, k, k, k, k), lambda: B.sablock_decode_paged(pages, k, k, k, k, k, k, k),
                 lambda: B.sablock_select_pages(pages, k, k, k, k, 3, k, k), lambda: B.sablock_compact_paged(_shape(), k, k, k, 3, True, pages, k, k, k)):
        with pytest.raises(ValueError, match="device memory"):  # before the library is asked
            call()


def test_decode_launches_as_the_plan_of_the_tests_says(tmp_path):
    # (dtype, D, problems, compute units): workgroups, rows alone, rows of a step that shares and of one that does not
    from paged_plan import launch

    cases = [(t, D, P, cus) for t in ("bf16", "f32") for D in (32, 64, 96, 128, 160, 192, 256) for P in (1, 255, 256, 4096) for cus in (4, 256, 400)]
    rows = _run_host_code(tmp_path, """
#include "paged_decode.hip"
#include <cstdio>
int main()
{
    for (const auto &c : std::initializer_list<std::array<int, 4>>{%s}) {
        sablock::PageDims d{};
        d.dtype = c[0]; d.D = c[1]; d.P = c[2]; d.cus = c[3];
        const bool bf = d.dtype == SABLOCK_BF16;
        std::printf("%%d %%d %%d %%d\\n", sablock::workgroups_of(d), sablock::rows_alone(d), sablock::step_rows(bf, d.D, false), sablock::step_rows(bf, d.D, true));
    }
}
""" % ", ".join("{%d, %d, %d, %d}" % (B.SABLOCK_BF16 if t == "bf16" else B.SABLOCK_F32, D, P, cus) for t, D, P, cus in cases), header="array")
    for (t, D, P, cus), (workgroups, rows_alone, shared, alone) in zip(cases, rows, strict=True):
        assert launch(t, D, P, cus, 1 << 17) == (workgroups, rows_alone, shared)
        assert launch(t, D, P, cus, 16) == (0, rows_alone, alone)

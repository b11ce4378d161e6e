"""Where the pieces of common prefixes lie in the workspace, as the kernels count them, and its size (host code, no GPU needed)."""

import ctypes

import pytest

from test_host_logic import _run_host_code, lib  # noqa: F401
from test_paged_host import FAKE, _pages

MANY = 4096


def test_places_of_any_prefixes_lie_in_the_workspace(tmp_path):
    # begins that ascend have no more pieces than the workspace has room for; of others each prefix may have nearly 2^30 by itself, and their sum passes 32 bits
    slots = [600, 98302 + 512, 229374]
    alls = [0, 1, 599, 4096, 524288, 2 ** 30 - 1]
    rows = _run_host_code(tmp_path, """
#include "paged_prefix.hip"
#include <cstdio>
int main()
{
    for (int slots : {%s})
        for (int all : {%s})
            for (int blocks : {1, 8}) {
                const int pieces = all / 8 / blocks;           // of a problem and block of columns, eight problems
                int32_t before = 0;
                bool wrapped = false;
                long outside = 0, refused = 0;
                for (int i = 0; i < %d; ++i) {
                    if (pieces)
                        for (int problem : {0, 7}) {
                            const int64_t at = before + (int64_t)problem * pieces * blocks + blocks - 1, last = at + (int64_t)(pieces - 1) * blocks;
                            const bool placed = sablock::have_places(at, pieces, blocks, slots);
                            refused += !placed;
                            outside += placed && (at < 0 || last >= slots);
                        }
                    wrapped |= __builtin_add_overflow(before, sablock::counted_pieces(all, slots), &before);
                }
                std::printf("%%d %%d %%d %%d %%ld %%ld\\n", slots, all, blocks, (int)wrapped, outside, refused);
            }
    std::printf("%%d %%d %%d\\n", (int)sablock::have_places(-1, 1, 1, 600), (int)sablock::have_places(-(1ll << 31), 4, 8, 600), (int)sablock::have_places(599, 1, 1, 600));
}
""" % (", ".join(map(str, slots)), ", ".join(map(str, alls)), MANY), "initializer_list")
    assert rows.pop() == [0, 0, 1]
    assert len(rows) == len(slots) * len(alls) * 2
    for room, all_, blocks, wrapped, outside, refused in rows:
        assert not wrapped and not outside, (room, all_, blocks)
        # those whose pieces fit in front of the end are placed, by exact sums
        pieces, want = all_ // 8 // blocks, 0
        for i in range(MANY if pieces else 0):
            for problem in (0, 7):
                at = i * all_ + problem * pieces * blocks + blocks - 1
                want += at + (pieces - 1) * blocks >= room
        assert refused == want, (room, all_, blocks)


# sequences, query and KV heads, elements, fp32, and the most prefixes that go by many columns: above 64 columns on average, 16 where heads have more than 128 elements
SHAPES = [(64, 32, 8, 128, False, 3), (64, 32, 8, 64, False, 3), (65, 8, 8, 128, False, 1), (64, 8, 8, 128, False, 0), (32, 32, 8, 256, False, 7), (200, 16, 1, 256, False, 199),
          (4096, 16, 1, 32, False, 1023), (64, 32, 8, 128, True, 0), (3, 2, 1, 160, False, 0)]


def _size(lib, pages, n):  # noqa: F811
    size = ctypes.c_size_t(0)
    assert lib.sablock_decode_prefix_paged_workspace_bytes(ctypes.byref(pages), n, ctypes.byref(size)) == 0
    return size.value


@pytest.mark.parametrize("n_seq,hq,hkv,D,f32,wide", SHAPES, ids=str)
def test_a_workspace_serves_calls_with_fewer_prefixes(lib, n_seq, hq, hkv, D, f32, wide):  # noqa: F811
    pages = _pages(n_seq=n_seq, n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=D, dtype=0 if f32 else 1,
                   k_stride=dict(enumerate([0, hkv * 16 * D, 16 * D, D])), v_stride=dict(enumerate([0, hkv * 16 * D, 16 * D, D])))
    sizes = [_size(lib, pages, n) for n in range(1, 4097)]
    assert sizes == sorted(sizes)
    # the call itself takes what its own number needs: less where its columns are few, and nothing less than that
    call = lambda n, size: lib.sablock_decode_prefix_paged(ctypes.byref(pages), *[FAKE] * 7, n, FAKE, FAKE, size, None)  # noqa: E731
    for n in {1, max(wide, 1), wide + 1, 64, 4096}:
        assert call(n, 0) == 3
        need = int(lib.sablock_last_error().decode().split("<")[1].split()[0])
        assert need <= sizes[n - 1] and call(n, need - 1) == 3
        assert need == sizes[n - 1] or n > wide > 0
        assert all(need <= x for x in sizes[n - 1:])

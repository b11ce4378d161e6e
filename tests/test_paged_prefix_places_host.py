"""Where the pieces of common prefixes lie in the workspace, as the kernels count them (host code, no GPU needed)."""

from test_host_logic import _run_host_code

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

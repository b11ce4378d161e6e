"""Decode attention of sequences that have their first pages in common, against the formula in 64 bits."""

import math

import numpy as np
import pytest

from test_gpu_paged import NAN, Cache, _ref_decode, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")
INT_MAX = 2 ** 31 - 1


class Sharing(Cache):
    """Sequences `own` rows behind the pages of their prefix; prefixes: (sequences, pages)."""

    def __init__(self, torch, seed, prefixes, own, **kw):
        page = kw.get("page", 16)
        behind = [m for count, m in prefixes for _ in range(count)]
        behind += [0] * (len(own) - len(behind))
        super().__init__(torch, seed, [n + m * page for n, m in zip(own, behind)], **kw)
        self.begin, self.counts = [0], [m for _, m in prefixes]
        for count, m in prefixes:
            first = self.begin[-1]
            self.table[first: first + count, :m] = self.table[first, :m].clone()
            self.begin.append(first + count)
        self.fill()

    def decode_prefix(self, q, begin=None, pages=None, ws_fill=0xFF):
        torch = self.torch
        begin, pages = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (begin or self.begin, pages or self.counts))
        ws = torch.full((self.B.sablock_decode_prefix_paged_workspace_bytes(self.pages, pages.numel()),), ws_fill, dtype=torch.uint8, device="cuda")
        out = torch.full(q.shape, NAN, dtype=torch.float32, device="cuda")
        self.B.sablock_decode_prefix_paged(self.pages, q, self.k_pool, self.v_pool, self.table, self.lengths, begin, pages, out, ws)
        return out


def _check(c, q, begin=None, pages=None, ref=None):
    got = c.decode_prefix(q, begin, pages).double().cpu()
    most = max(float(c.rows(c.v_pool, s).abs().max()) if int(c.lengths[s]) > 0 else 0.0 for s in range(c.n))
    err = (got - (_ref_decode(c, q) if ref is None else ref)).abs().max()
    # as in the test of the attention without prefixes; one more product and sum for what is joined
    assert err <= 2.0 ** -16 * max(most, 1.0), float(err)
    return got


HEADS = [(1, 32, "bf16", 16), (2, 64, "bf16", 32), (3, 96, "bf16", 16), (4, 128, "bf16", 16), (4, 128, "bf16", 64), (5, 160, "bf16", 128), (7, 192, "bf16", 16), (8, 224, "bf16", 256),
         (16, 128, "bf16", 16), (12, 256, "bf16", 32), (1, 16, "f32", 16), (4, 64, "f32", 64), (7, 80, "f32", 16), (16, 128, "f32", 32), (5, 240, "f32", 128), (9, 256, "f32", 16)]


@pytest.mark.parametrize("G,D,dtype,page", HEADS)
@pytest.mark.parametrize("prefixes,own", [([(2, 1)], [1, 0]), ([(3, 7)], [5, 0, 40]), ([(5, 3), (2, 20)], [0, 1, 15, 16, 17, 300, 33]), ([(9, 40)], [3, 700, 0, 1, 2, 64, 5, 20, 9]),
                                          ([(2, 2), (1, 30), (4, 1)], [3, 4, 5, 6, 7, 8, 9, 100, 0])], ids=str)
def test_groups_heads_pages_and_lengths(torch_cuda, G, D, dtype, page, prefixes, own):  # noqa: F811
    torch = torch_cuda
    # pages of 256 rows are many rows
    prefixes = [(n, m if page <= 64 else -(-m // 4)) for n, m in prefixes]
    c = Sharing(torch, G * D + len(own), prefixes, own, layers=2, heads=2, group=G, D=D, dtype=dtype, page=page, k_axes=(1, 2, 0, 3), pad=16)
    _check(c, c.normal((c.n, 2, 2 * G, D)))


@pytest.mark.parametrize("G,D,dtype,page,count,pages,heads", [(4, 128, "bf16", 16, 40, 150, 2), (7, 64, "bf16", 32, 30, 40, 3), (16, 256, "bf16", 16, 9, 120, 1), (1, 96, "bf16", 16, 200, 60, 1),
                                                              (5, 64, "f32", 16, 33, 80, 2), (2, 128, "f32", 64, 50, 12, 1), (4, 128, "bf16", 128, 129, 9, 2), (8, 32, "bf16", 16, 300, 30, 1),
                                                              (3, 256, "bf16", 64, 30, 50, 2), (8, 256, "bf16", 256, 21, 5, 1), (2, 256, "bf16", 16, 70, 33, 2),
                                                              (4, 160, "bf16", 16, 40, 33, 2), (3, 192, "bf16", 64, 27, 12, 2), (8, 224, "bf16", 32, 17, 40, 1)])
def test_many_sequences(torch_cuda, G, D, dtype, page, count, pages, heads):  # noqa: F811
    # several blocks of columns, the last one short; sequences that end at their prefix, in front of it, or have nothing
    torch = torch_cuda
    own = [(s * 37) % 90 for s in range(count)]
    c = Sharing(torch, count, [(count, pages)], own, heads=heads, group=G, D=D, dtype=dtype, page=page)
    short = {0: 0, 1: 5, 2: pages * page - 1, count // 2: pages * page, count - 1: page}
    for s, n in short.items():
        c.lengths[s] = n
    c.table[0, :pages] = -1                                     # has no row, nor pages
    q = c.normal((c.n, 1, heads * G, D))
    got = _check(c, q)
    assert not got[0].any()


@pytest.mark.parametrize("n_prefixes,dtype,D", [(64, "bf16", 128), (65, "bf16", 64), (150, "f32", 64), (400, "bf16", 32)])
def test_many_prefixes(torch_cuda, n_prefixes, dtype, D):  # noqa: F811
    # more than a wavefront has lanes; of one sequence, of none, and without pages among them
    torch = torch_cuda
    rng = np.random.default_rng(n_prefixes)
    prefixes = [(int(rng.integers(0, 5)), int(rng.integers(0, 9)) if i % 13 else 70) for i in range(n_prefixes)]
    n = sum(x for x, _ in prefixes) + 2                         # two behind the last prefix
    own = [int(rng.integers(0, 60)) for _ in range(n)]
    page = 16
    behind = [m for count, m in prefixes for _ in range(count)] + [0, 0]
    c = Cache(torch, n, [a + m * page for a, m in zip(own, behind)], heads=1, group=2, D=D, dtype=dtype, page=page)
    c.__class__ = Sharing
    c.begin, c.counts = [0], [m for _, m in prefixes]
    for count, m in prefixes:
        first = c.begin[-1]
        if count:
            c.table[first: first + count, :m] = c.table[first, :m].clone()
        c.begin.append(first + count)
    c.k_pool.copy_(c.normal(c.k_pool.shape))
    c.v_pool.copy_(c.normal(c.v_pool.shape))
    _check(c, c.normal((n, 1, 2, D)))


@pytest.mark.parametrize("G,D,dtype,page", [(4, 128, "bf16", 16), (7, 64, "bf16", 128), (16, 256, "bf16", 32), (3, 64, "f32", 16), (8, 256, "f32", 64)])
@pytest.mark.parametrize("count,rows,own", [(2, 16, 1), (3, 3000, 1000), (40, 5000, 0), (70, 800, 40)])
def test_every_row_counts_once(torch_cuda, G, D, dtype, page, count, rows, own):  # noqa: F811
    # equal logits: the mean of V.  V[r] = 1 in column r % D and 0 elsewhere, so a row that is lost, or comes twice, shows as a share of 1 / length.
    # 2^-20 relative for the quotients and the sums of whole numbers
    torch = torch_cuda
    pages = -(-rows // page)
    c = Sharing(torch, rows, [(count, pages)], [own + s % 3 for s in range(count)], heads=1, group=G, D=D, dtype=dtype, page=page)
    want = torch.empty((count, D), dtype=torch.float64, device="cuda")
    for s, n in enumerate(c.lengths.tolist()):
        r = torch.arange(n, device="cuda")
        ids = c.table[s, r // page].long()
        c.k_pool[0, ids, 0, r % page] = 0.0
        one = torch.nn.functional.one_hot(r % D, D).to(c.dt)
        c.v_pool[0, ids, 0, r % page] = one
        want[s] = one.double().mean(dim=0)
    got = c.decode_prefix(c.normal((count, 1, G, D))).double()
    assert torch.allclose(got, want[:, None, None].expand_as(got), rtol=2.0 ** -20, atol=0)


def test_begins_and_pages_out_of_range(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Sharing(torch, 3, [(5, 6)], [10, 300, 0, 4, 90], heads=2, group=2, D=64)
    q = c.normal((5, 1, 4, 64))
    ref = _ref_decode(c, q)
    for begin, pages in (([0, 5], [6]), ([-7, 5], [6]), ([0, INT_MAX], [6]), ([0, 5], [3]), ([0, 5], [-4]), ([0, 0], [6]), ([2, 4], [6]), ([0, 2, 2, 5], [6, 100, 4]), ([3, 4, 5], [6, 6]),
                         ([-2 ** 31, -5, 3, INT_MAX], [INT_MAX, 6, 5]), ([5, 5], [6]), ([9, 12], [6])):
        _check(c, q, begin, pages, ref)
    # pages that no sequence has all of: each is read by itself
    for pages in ([26], [INT_MAX]):
        _check(c, q, [0, 5], pages, ref)
    # prefixes that do not follow each other: some result, of finite numbers, and no more
    for begin in ([5, 0], [0, 5, 0, 5, 0, 5], [3, 1, 4, 1, 5]):
        assert c.decode_prefix(q, begin, [6] * (len(begin) - 1), 0).shape == q.shape


def test_pages_of_a_prefix_that_do_not_exist(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Sharing(torch, 5, [(4, 12)], [0, 20, 33, 5], heads=2, group=2, D=64)
    q = c.normal((4, 1, 4, 64))
    full = c.table.clone()
    c.table[:, 3], c.table[:, 10], c.table[1, 12] = -1, c.n_pages, INT_MAX
    got = c.decode_prefix(q).double().cpu()
    for s, n in enumerate(c.lengths.tolist()):
        gone = {3, 10} | ({12} if s == 1 else set())
        keep = torch.tensor([r for r in range(n) if r // 16 not in gone])
        now, c.table = c.table, full
        k, v = c.rows(c.k_pool, s)[0][:, keep], c.rows(c.v_pool, s)[0][:, keep]
        c.table = now
        for h in range(2):
            x = torch.softmax(q[s, 0, 2 * h: 2 * h + 2].double().cpu() @ k[h].T / math.sqrt(64), dim=-1) @ v[h]
            assert bool(((got[s, 0, 2 * h: 2 * h + 2] - x).abs() <= 2.0 ** -16 * 5).all())
    c.table[:, :12] = -1                                        # none exists: the own rows alone, zeros without any
    got = c.decode_prefix(q).double().cpu()
    assert not got[0].any() and not torch.isnan(got).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["prefix", "own"])
def test_values_and_rows_that_are_no_number(torch_cuda, dtype, where):  # noqa: F811
    # in the prefix: of all that have it; in own rows, or a query: of that sequence alone
    torch = torch_cuda
    c = Sharing(torch, 6, [(3, 10), (2, 4)], [20, 30, 40, 10, 60], heads=2, group=2, D=64, dtype=dtype)
    c.lengths[2] = 70                                           # takes no part: its rows are those of four pages and six rows
    q = c.normal((5, 1, 4, 64))
    clean = c.decode_prefix(q)
    row = 100 if where == "prefix" else 165
    c.v_pool[0, int(c.table[1, row // 16]), 0, row % 16, 3] = INF
    c.k_pool[0, int(c.table[1, row // 16]), 1, row % 16, 3] = NAN
    got = c.decode_prefix(q)
    hit = [0, 1] if where == "prefix" else [1]
    assert bool((got[hit][:, 0, :2, 3] == INF).all()) and bool(torch.isnan(got[hit][:, 0, 2:]).all())
    got[hit, 0, :2, 3], got[hit, 0, 2:] = clean[hit, 0, :2, 3], clean[hit, 0, 2:]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("late", [5.0, 200.0, -300.0])
def test_logits_that_rise_between_the_prefix_and_the_own_rows(torch_cuda, dtype, late):  # noqa: F811
    torch = torch_cuda
    D = 64
    c = Sharing(torch, 9, [(4, 100)], [400, 0, 1, 50], heads=1, group=3, D=D, dtype=dtype)
    c.k_pool.zero_()
    for s, n in enumerate(c.lengths.tolist()):
        r = torch.arange(1600 if late != 5.0 else 800, n, device="cuda")
        if len(r):
            c.k_pool[0, c.table[s, r // 16].long(), 0, r % 16, 0] = late
    q = torch.zeros((4, 1, 3, D), device="cuda")
    q[..., 0] = D ** 0.5
    got, ref = c.decode_prefix(q.to(c.dt)).double().cpu(), _ref_decode(c, q.to(c.dt))
    assert bool(((got - ref).abs() <= 2.0 ** -15 * 6).all())    # logits up to 2^8.8 in the log2 domain: 2^-16 in a share


def test_twice_the_same_on_any_stream_and_in_a_graph(torch_cuda):  # noqa: F811
    # equal bits whatever the workspace holds; a graph whose lengths, table and prefixes change between replays
    torch = torch_cuda
    c = Sharing(torch, 12, [(6, 60), (3, 5)], [30, 0, 200, 9, 1, 77, 400, 20, 3, 50], layers=2, heads=2, group=4, D=128)
    q = c.normal((10, 2, 8, 128))
    want = c.decode_prefix(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for fill in (0, 0xFF, 0x7F):
        with torch.cuda.stream(side):
            again = c.decode_prefix(q, ws_fill=fill)
        side.synchronize()
        assert torch.equal(again, want)
    begin, pages = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (c.begin, c.counts))
    ws = torch.empty((c.B.sablock_decode_prefix_paged_workspace_bytes(c.pages, 2),), dtype=torch.uint8, device="cuda")
    out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.B.sablock_decode_prefix_paged(c.pages, q, c.k_pool, c.v_pool, c.table, c.lengths, begin, pages, out, ws)
    for b, m, lengths in ((c.begin, c.counts, None), ([0, 4, 6], [60, 30], None), ([0, 6, 9], [59, 5], 970), ([6, 9, 9], [5, 5], 0)):
        begin.copy_(torch.tensor(b, dtype=torch.int32))
        pages.copy_(torch.tensor(m, dtype=torch.int32))
        if lengths is not None:
            c.lengths[2] = lengths
        q.copy_(c.normal(q.shape))
        eager = c.decode_prefix(q, b, m)
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        _check(c, q, b, m)


@pytest.mark.parametrize("dtype,G,count", [("bf16", 8, 4), ("bf16", 8, 40), ("f32", 8, 4)])
def test_probabilities_are_fp32(torch_cuda, dtype, G, count):  # noqa: F811
    # As in the test of the attention without prefixes: three rows whose logits are exact products, here the prefix's, whose other rows have no share.  The
    # shares' sum to 2^-19, each share to 2^-19.7 and 2^-19, and for what the join multiplies and divides, four roundings more, 2^-22
    torch = torch_cuda
    D, n = 64, 6 * count
    c = Sharing(torch, 1, [(count, 1)] * 6, [0] * n, heads=1, group=G, D=D, dtype=dtype)
    at = c.table[::count, 0].long()
    first = (torch.rand((6, 3), generator=c.gen, device="cuda") * 2 - 1).to(torch.bfloat16)
    c.k_pool[0, at, 0] = 0.0
    c.k_pool[0, at, 0, :, 0] = -1e6
    c.k_pool[0, at, 0, :3, 0] = first.to(c.dt)
    c.v_pool[0, at, 0] = 0.0
    c.v_pool[0, at, 0, :3, 0] = 1.0
    for r in range(3):
        c.v_pool[0, at, 0, r, 1 + r] = 1.0
    q = torch.zeros((n, 1, G, D), dtype=c.dt, device="cuda")
    q[..., 0] = torch.arange(1, G + 1, device="cuda").to(c.dt)
    got = c.decode_prefix(q)[:, 0].double().cpu()
    share = torch.softmax(first.double().cpu()[:, None] * torch.arange(1, G + 1, dtype=torch.float64)[:, None] / 8, dim=-1).repeat_interleave(count, dim=0)
    assert bool(((got[..., 0] - 1).abs() <= 2.0 ** -19 + 2.0 ** -22).all()), float((got[..., 0] - 1).abs().max())
    assert bool(((got[..., 1:4] - share).abs() <= (2.0 ** -19.7 + 2.0 ** -19 + 2.0 ** -22) * share).all())
    assert not got[..., 4:].any()

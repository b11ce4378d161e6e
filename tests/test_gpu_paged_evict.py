"""Eviction from the paged cache by gathered weight, against sorted lists and copies on the host, bit for bit."""

import pytest

from test_gpu_paged import GARBAGE, NAN, Cache, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")


def _bits(t):
    return t.contiguous().view({2: __import__("torch").int16, 4: __import__("torch").int32}[t.element_size()])


class Evictable(Cache):
    """A cache with weights, and a second table of pages that no row lies in."""

    def __init__(self, torch, seed, lengths, keep, capacity=None, **kw):
        longest = max(max(lengths), 1)
        page = kw.get("page", 16)
        cap = longest if capacity is None else capacity
        news = [-(-min(max(n, 0), keep) // page) for n in lengths]
        super().__init__(torch, seed, [max(0, min(n, cap)) for n in lengths], spare=sum(news) + 2, **kw)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        wide = -(-cap // page)
        if wide > self.width:
            self.table = torch.cat([self.table, torch.full((self.n, wide - self.width), -7, dtype=torch.int32, device="cuda")], dim=1)
        self.width = self.table.shape[1]
        used = set(self.table[self.table >= 0].tolist())
        free = [i for i in range(self.n_pages) if i not in used]
        self.after = torch.full_like(self.table, -1)
        at = 0
        for s, m in enumerate(news):
            m = min(m, self.width)
            self.after[s, :m] = torch.tensor(free[at: at + m], dtype=torch.int32, device="cuda")
            at += m
        self.pages = self.B.make_pages(self.k_pool, self.v_pool, self.table, self.H * self.G)
        self.weights = torch.randn((self.L, self.n_pages, self.H, page), generator=self.gen, device="cuda")
        self.keep = keep

    def randomise(self):
        """Ordinary numbers everywhere: rows are only copied here."""
        for t in (self.k_pool, self.v_pool):
            t.copy_(self.normal(t.shape))
        return self

    def evict(self, first, last, fill=0xFF, **kw):
        torch = self.torch
        ws = torch.full((self.B.sablock_evict_paged_workspace_bytes(self.pages),), fill, dtype=torch.uint8, device="cuda")
        self.len_out = torch.full((self.n,), -5, dtype=torch.int32, device="cuda")
        self.rows_out = torch.full((self.n * self.L * self.H, self.keep), -99, dtype=torch.int32, device="cuda")
        self.B.sablock_evict_paged(self.pages, self.table, self.lengths, self.weights, self.k_pool, self.v_pool, self.keep, self.after, self.len_out, self.rows_out,
                                   ws, n_first=first, n_last=last, bounds=self.bounds, **kw)


def _key(w):
    return INF if w != w else w


def _ref_rows(c, weights, first, last):
    """The rows that stay, per problem; a weight that is no number in front of infinity, pages that do not exist behind everything."""
    lists = []
    cap = c.width * c.page
    for s in range(c.n):
        n = min(max(int(c.lengths[s]), 0), cap)
        ids = c.table[s, : -(-n // c.page)].tolist()
        for l in range(c.L):
            for h in range(c.H):
                if n <= c.keep:
                    lists.append(list(range(n)))
                    continue
                w = [float(weights[l, ids[r // c.page], h, r % c.page]) if 0 <= ids[r // c.page] < c.n_pages else -INF for r in range(n)]
                forced = set(range(first)) | set(range(n - last, n))
                rest = sorted((r for r in range(n) if r not in forced), key=lambda r: (0 if w[r] != w[r] else 1, -_key(w[r]), r))
                lists.append(sorted(list(forced) + rest[: c.keep - len(forced)]))
    return lists


def _check(c, first, last):
    torch = c.torch
    was = [t.clone() for t in (c.k_pool, c.v_pool, c.weights, c.bounds)]
    c.evict(first, last)
    lists = _ref_rows(c, was[2].cpu(), first, last)
    assert c.rows_out.tolist() == [x + [-1] * (c.keep - len(x)) for x in lists]
    cap = c.width * c.page
    assert c.len_out.tolist() == [min(max(int(n), 0), cap, c.keep) for n in c.lengths.tolist()]
    want = [t.clone() for t in was]
    for p, rows in enumerate(lists):
        s, l, h = p // (c.L * c.H), p // c.H % c.L, p % c.H
        r, j = torch.tensor(rows, dtype=torch.long, device="cuda"), torch.arange(len(rows), device="cuda")
        source, dest = c.table[s].long()[r // c.page], c.after[s].long()[j // c.page]
        ok = (source >= 0) & (source < c.n_pages)
        there = (dest >= 0) & (dest < c.n_pages)
        for old, new in zip(was[:3], want[:3]):
            x = old[l, source.clamp(0, c.n_pages - 1), h, r % c.page]
            x = torch.where(ok.view([-1] + [1] * (x.dim() - 1)), x, torch.zeros((), dtype=x.dtype, device="cuda"))
            new[l, dest[there], h, (j % c.page)[there]] = x[there]
        for i in range(-(-len(rows) // c.page)):
            at = int(c.after[s, i])
            if 0 <= at < c.n_pages:
                held = want[0][l, at, h, : min(c.page, len(rows) - i * c.page)].float()
                want[3][l, at, h, 0], want[3][l, at, h, 1] = held.amin(dim=0), held.amax(dim=0)
    for got, ref in zip((c.k_pool, c.v_pool, c.weights), want):
        assert torch.equal(_bits(got), _bits(ref))             # and everything else as it was
    assert torch.equal(torch.nan_to_num(c.bounds.float(), 7.0), torch.nan_to_num(want[3].float(), 7.0))
    return lists


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f32", 64)])
def test_sequences_that_stay_where_they_are(torch_cuda, dtype, page):  # noqa: F811
    # the old entries of those that keep all their rows: pages that two of them share as well; the others' rows move
    torch = torch_cuda
    c = Evictable(torch, 21, [100, 300, 90, 0, 128, 77], 128, layers=2, heads=2, group=2, D=64, dtype=dtype, page=page).randomise()
    for s in (0, 2, 4):
        c.after[s] = c.table[s]
    c.table[2, 0] = c.after[2, 0] = c.table[0, 0]
    before = c.table.clone()
    was = [t.clone() for t in (c.k_pool, c.v_pool, c.weights)]
    c.evict(4, 16)
    assert c.len_out.tolist() == [100, 128, 90, 0, 128, 77] and torch.equal(c.table, before)
    lists = _ref_rows(c, was[2].cpu(), 4, 16)
    assert c.rows_out.tolist() == [x + [-1] * (c.keep - len(x)) for x in lists]
    held = {int(c.table[s, i]): min(page, n - i * page) for s, n in ((0, 100), (2, 90), (4, 128)) for i in range(-(-n // page))}
    stay = sorted(held)
    for at, m in held.items():
        rows = c.k_pool[:, at, :, :m].float()
        assert torch.equal(c.bounds[:, at, :, 0].float(), rows.amin(dim=2)) and torch.equal(c.bounds[:, at, :, 1].float(), rows.amax(dim=2))
    for got, old in zip((c.k_pool, c.v_pool, c.weights), was):
        assert torch.equal(got[:, stay], old[:, stay])
        for p, rows in enumerate(lists):
            s, l, h = p // 4, p // 2 % 2, p % 2
            for j, r in enumerate(rows):
                assert torch.equal(got[l, int(c.after[s, j // page]), h, j % page], old[l, int(c.table[s, r // page]), h, r % page])


@pytest.mark.parametrize("D,dtype,page", [(8, "f32", 16), (64, "bf16", 16), (96, "bf16", 32), (128, "bf16", 64), (256, "bf16", 256), (256, "f32", 16), (40, "bf16", 128)])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 0, 1), (17, 1, 1), (64, 4, 16), (100, 0, 50), (300, 150, 150), (400, 3, 0)])
def test_evict(torch_cuda, D, dtype, page, keep, first, last):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, D + keep, [0, 1, 17, 301, 400, 640], keep, layers=2, heads=3, group=1, D=D, dtype=dtype, page=page, k_axes=(1, 0, 3, 2), pad=8).randomise()
    _check(c, first, last)


@pytest.mark.parametrize("rows,capacity,keep", [(4096, 4096, 1000), (4097, 5000, 4096), (9000, 16384, 2000), (20000, 20000, 128), (3000, 140000, 2500), (140001, 140016, 40000)])
def test_evict_from_long_sequences(torch_cuda, rows, capacity, keep):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, keep, [rows, 3, rows // 2], keep, capacity=capacity, heads=2, group=1, D=8).randomise()
    _check(c, 4, keep // 4)


def test_equal_weights_and_what_is_no_number(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, 3, [500], 40, heads=1, group=1, D=16).randomise()
    c.weights.zero_()
    assert _check(c, 2, 8)[0] == list(range(32)) + list(range(492, 500))
    place = lambda r: (0, int(c.table[0, r // 16]), 0, r % 16)  # noqa: E731
    c.weights[place(100)], c.weights[place(200)], c.weights[place(150)] = NAN, INF, NAN
    c.weights[place(5)], c.weights[place(6)], c.weights[place(7)] = -INF, -0.0, -1e-38
    rows = _check(c, 0, 0)[0]
    assert {100, 200, 150, 6} < set(rows) and 5 not in rows and 7 not in rows
    c.keep = 2
    assert _check(c, 0, 0)[0] == [100, 150]
    c.weights.fill_(-INF)
    assert _check(c, 0, 1)[0] == [0, 499]


def test_pages_that_do_not_exist(torch_cuda):  # noqa: F811
    # old ones: their rows go first, or stay as rows of zeros; new ones: what would go there is dropped
    torch = torch_cuda
    c = Evictable(torch, 4, [200, 64, 300], 100, heads=2, group=2, D=64, dtype="f32").randomise()
    c.table[0, 2], c.table[0, 12], c.table[1, 1], c.table[2, 3] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    c.after[2, 1], c.after[2, 6] = c.n_pages, -3
    lists = _check(c, 1, 10)
    assert 40 not in lists[0] and 195 in lists[0] and len(lists[2]) == 64


def test_lengths_that_the_table_does_not_hold(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, 5, [160, 160, 160], 70, heads=2, group=1, D=32).randomise()
    c.table = c.table[:, :10].contiguous()
    c.after = c.after[:, :10].contiguous()
    c.width = 10
    c.pages = c.B.make_pages(c.k_pool, c.v_pool, c.table, 2)
    c.lengths = torch.tensor([-4, 2 ** 31 - 1, 161], dtype=torch.int32, device="cuda")
    _check(c, 1, 5)


def test_sequences_that_share_their_first_pages(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, 6, [400, 320, 336], 120, heads=2, group=2, D=64, page=16).randomise()
    c.table[1, :15] = c.table[0, :15]
    c.table[2, :15] = c.table[0, :15]
    _check(c, 4, 30)


def test_garbage_behind_the_rows_does_not_matter(torch_cuda):  # noqa: F811
    # the pools and weights behind a sequence's last row hold anything; without bounds, on another stream, twice the same
    torch = torch_cuda
    c = Evictable(torch, 7, [333, 90], 64, heads=2, group=1, D=64).randomise()
    last = int(c.table[0, 333 // 16])
    c.weights[:, last, :, 333 % 16:] = torch.tensor(GARBAGE[:3], device="cuda")
    c.k_pool[:, last, :, 333 % 16:] = NAN
    bounds, c.bounds = c.bounds, None
    was = c.k_pool.clone()
    c.evict(2, 9)
    rows, k = c.rows_out.clone(), c.k_pool.clone()
    assert rows.cpu().tolist() == [x + [-1] * (64 - len(x)) for x in _ref_rows(c, c.weights.cpu(), 2, 9)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for fill in (0, 0x7F):
        with torch.cuda.stream(side):
            c.k_pool.copy_(was)
            c.evict(2, 9, fill)
        side.synchronize()
        assert torch.equal(c.rows_out, rows) and torch.equal(_bits(c.k_pool), _bits(k))
    assert bounds is not None


def test_evict_captured_and_replayed(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Evictable(torch, 8, [500, 130, 260], 128, layers=2, heads=2, group=1, D=64).randomise()
    ws = torch.empty((c.B.sablock_evict_paged_workspace_bytes(c.pages),), dtype=torch.uint8, device="cuda")
    c.evict(4, 32)
    rows = torch.empty_like(c.rows_out)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.B.sablock_evict_paged(c.pages, c.table, c.lengths, c.weights, c.k_pool, c.v_pool, 128, c.after, c.len_out, rows, ws, n_first=4, n_last=32, bounds=c.bounds)
    for rep in range(3):
        c.weights.copy_(torch.randn(c.weights.shape, generator=c.gen, device="cuda"))
        c.lengths.copy_(torch.tensor([500 - rep, 130, 128 + rep], dtype=torch.int32, device="cuda"))
        eager_weights = c.weights.clone()
        c.evict(4, 32)
        want = [t.clone() for t in (c.rows_out, c.k_pool, c.v_pool, c.weights, c.bounds, c.len_out)]
        c.weights.copy_(eager_weights)
        rows.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((rows, c.k_pool, c.v_pool, c.weights, c.bounds, c.len_out), want):
            assert torch.equal(torch.nan_to_num(got.float(), 7.0), torch.nan_to_num(ref.float(), 7.0)), rep

"""Attention with common pages where the columns are many (K and V in LDS, every wavefront with columns of its own), at its odd places, against the formula in 64 bits."""

import math

import pytest

from test_gpu_paged import NAN, torch_cuda  # noqa: F401
from test_gpu_paged_prefix import INF, INT_MAX, Sharing

pytestmark = pytest.mark.gpu

# group, head elements, page, sequences, KV heads
SHAPES = [(8, 64, 16, 20, 2), (4, 128, 64, 40, 1), (8, 96, 16, 33, 1), (4, 256, 16, 10, 2), (5, 160, 64, 9, 1), (16, 32, 32, 9, 1), (3, 224, 16, 30, 1)]
FEW = 8                                        # compute units that the plan is made for: pieces of many steps


def _is_wide(G, D, n_seq, n_prefixes):
    """The launch's rule: more than 64 columns of a prefix on average, 16 where heads have more than 128 elements."""
    return n_seq * G > (64 if D <= 128 else 16) * n_prefixes


def _batch(torch, shape, pages, seed=1, units=FEW, own=None):
    G, D, page, n, heads = shape
    assert _is_wide(G, D, n, 1)
    c = Sharing(torch, seed, [(n, pages)], [(s * 37) % 90 for s in range(n)] if own is None else own, heads=heads, group=G, D=D, page=page, spare=5)
    if units:
        c.pages.compute_units = units
    # page 0, which is read in the place of those that do not exist, is nobody's
    spare = min(set(range(1, c.n_pages)) - set(c.table.flatten().tolist()))
    c.k_pool[:, spare], c.v_pool[:, spare] = c.k_pool[:, 0].clone(), c.v_pool[:, 0].clone()
    c.table[c.table == 0] = spare
    c.k_pool[:, 0], c.v_pool[:, 0] = NAN, INF
    return c


def _ref(c, q, rows=None):
    """Outputs in 64 bits on the GPU; rows(s): those of sequence s that count, all of them if not given."""
    torch = c.torch
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(c.lengths.tolist()):
        r = torch.arange(n, device="cuda")
        if rows is not None:
            r = r[rows(s, r)]
        if not len(r):
            continue
        ids = c.table[s].long()[r // c.page]
        for h in range(c.H):
            at = slice(h * c.G, (h + 1) * c.G)
            k, v = (x[0, ids, h, r % c.page].double() for x in (c.k_pool, c.v_pool))
            out[s, 0, at] = torch.softmax((q[s, 0, at].double() @ k.t().contiguous()) / math.sqrt(c.D), dim=-1) @ v
    return out


def _most(c):
    """The largest value of the sequences' rows: what lies behind them is not finite, or above 10^38."""
    v = c.v_pool[:, c.table[(c.table >= 0) & (c.table < c.n_pages)].unique().long()].float().abs()
    return float(v[v < 1e38].max())


def _close(c, got, want, most):
    # as in the test of the attention without prefixes: fp32 logits of up to 64 in the log2 domain
    err = (got.double() - want).abs().max()
    assert float(err) <= 2.0 ** -16 * max(most, 1.0), float(err)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("units", [FEW, 0])
def test_pages_that_do_not_exist(torch_cuda, shape, units):  # noqa: F811
    # the first, the last and middle ones of a prefix, one half of a step of 32 rows or all of it, whole pieces of them; own ones, too
    torch = torch_cuda
    G, D, page, n, heads = shape
    pages = 2400 // page + 1
    c = _batch(torch, shape, pages, units=units)
    q = c.normal((n, 1, heads * G, D))
    most, full = _most(c), c.table.clone()
    per = max(1, 32 // page)
    for gone in ([0], [pages - 1], [pages - 2], [1, pages // 2], [0, 1, 2, 3], list(range(per * 5, per * 6)), list(range(pages // 3, 2 * pages // 3)),
                 list(range(0, pages, 2)), list(range(1, pages, 2)), list(range(pages // 2, pages)), list(range(pages // 2)), list(range(pages))):
        c.table.copy_(full)
        for i, at in enumerate(gone):
            c.table[:, at] = (-1, c.n_pages, INT_MAX, -2 ** 31)[i % 4]
        c.table[3, pages] = -1                                  # 21 or more own rows of this one
        lost = torch.zeros(pages + 16, dtype=torch.bool, device="cuda")
        lost[gone] = True
        _close(c, c.decode_prefix(q), _ref_there(c, q, lost, pages), most)


def _ref_there(c, q, lost, pages):
    now = c.table
    c.table = now.clamp(0, c.n_pages - 1)
    ref = _ref(c, q, lambda s, r: ~(lost[r // c.page] | ((s == 3) & (r // c.page == pages))))
    c.table = now
    return ref


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("units", [FEW, 0])
def test_logits_that_rise_late(torch_cuda, shape, units):  # noqa: F811
    # step by step through every piece, at the very last row of the prefix, and behind it; half of the heads see them fall
    torch = torch_cuda
    G, D, page, n, heads = shape
    pages = 3200 // page + 1
    c = _batch(torch, shape, pages, units=units)
    c.k_pool.zero_()
    rows = pages * page
    r = torch.arange(rows, device="cuda")
    ids = c.table[0].long()[r // page]
    q = torch.zeros((n, 1, heads * G, D), dtype=c.dt, device="cuda")
    q[..., 0] = (torch.arange(heads * G, device="cuda") % 2 * 2 - 1).to(c.dt) * (D ** 0.5 // 1)
    most = _most(c)
    for ramp, last, own in ((0.0, 40.0, 0.0), (40.0 / rows, 0.0, 0.0), (40.0 / rows, 41.0, 42.0), (-40.0 / rows, -41.0, 0.0), (0.0, 0.0, 40.0), (0.0, -40.0, -40.0)):
        value = ramp * r
        if last:
            value[-1] = last
        c.k_pool[0, ids, :, r % page, 0] = value.to(c.dt)[:, None]
        for s, m in enumerate(c.lengths.tolist()):
            x = torch.arange(rows, m, device="cuda")
            c.k_pool[0, c.table[s].long()[x // page], :, x % page, 0] = own
        _close(c, c.decode_prefix(q), _ref(c, q), most)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_values_and_rows_that_are_no_number(torch_cuda, shape):  # noqa: F811
    # of a prefix: of all that have it, and one KV head's; of own rows or a query: of that sequence alone, the columns beside it as they were, bit for bit
    torch = torch_cuda
    G, D, page, n, heads = shape
    pages = 1600 // page + 1
    c = _batch(torch, shape, pages)
    c.lengths[2] = page + 5                                     # takes no part
    q = c.normal((n, 1, heads * G, D))
    clean = c.decode_prefix(q)
    members = [s for s in range(n) if s != 2]
    was = c.k_pool.clone(), c.v_pool.clone()

    def at(s, row):
        return 0, int(c.table[s, row // page]), heads - 1, row % page

    head = slice((heads - 1) * G, heads * G)
    for row in (page + 5, 3 * page + 2, 777, pages * page - 1):
        c.v_pool[at(0, row)][3] = INF
        c.v_pool[at(0, row)][D - 1] = -INF
        got, want = c.decode_prefix(q), clean.clone()
        want[members, 0, head, 3], want[members, 0, head, D - 1] = INF, -INF
        assert torch.equal(got, want), row
        c.v_pool.copy_(was[1])
        c.k_pool[at(0, row)][3] = NAN
        got = c.decode_prefix(q)
        assert bool(torch.isnan(got[members][:, 0, head]).all()), row
        got[members, 0, head] = clean[members, 0, head]
        assert torch.equal(got, clean), row
        c.k_pool.copy_(was[0])
        # infinity: no number where the query's element is positive, no share of the row where it is negative
        c.k_pool[at(0, row)][3] = INF
        got, up = c.decode_prefix(q), (q[..., 3] > 0)
        seen = torch.zeros_like(up)
        seen[members, 0, head] = True
        assert bool(torch.isnan(got[seen & up]).all()) and bool(torch.isfinite(got[~(seen & up)]).all())
        k = c.k_pool
        c.k_pool = was[0]
        ref = _ref(c, q, lambda s, r: r != row)
        c.k_pool = k
        down = seen & ~up
        assert bool(((got.double() - ref)[down].abs() <= 2.0 ** -16 * _most(c)).all())
        got[seen] = clean[seen]
        assert torch.equal(got, clean)
        c.k_pool.copy_(was[0])
    x = 5
    own = pages * page + 1
    c.v_pool[at(x, own)][7] = INF
    got, want = c.decode_prefix(q), clean.clone()
    want[x, 0, head, 7] = INF
    assert torch.equal(got, want)
    c.v_pool.copy_(was[1])
    for bad in (NAN, INF, -INF):
        was_q = q[x, 0, 1, 2].clone()
        q[x, 0, 1, 2] = bad
        got = c.decode_prefix(q)
        assert bool(torch.isnan(got[x, 0, 1]).all())            # keys of both signs: infinite logits of both signs, or none that is a number
        got[x, 0, 1] = clean[x, 0, 1]
        assert torch.equal(got, clean)
        q[x, 0, 1, 2] = was_q


@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
def test_begins_and_pages_out_of_range(torch_cuda, shape):  # noqa: F811
    torch = torch_cuda
    G, D, page, n, heads = shape
    c = _batch(torch, shape, 12, units=0)
    q = c.normal((n, 1, heads * G, D))
    ref, most = _ref(c, q), _most(c)
    for begin, pages in (([0, n], [12]), ([-7, n], [12]), ([0, INT_MAX], [12]), ([-2 ** 31, INT_MAX], [5]), ([0, n], [-4]), ([0, 0], [12]), ([1, n - 1], [12]), ([n - 2, n + 9], [12]),
                         ([n, n], [12]), ([n + 4, n + 9], [12]), ([n, 0], [12]), ([0, n], [INT_MAX]), ([0, n], [0]), ([3, 4], [12])):
        assert _is_wide(G, D, n, len(pages))
        _close(c, c.decode_prefix(q, begin, pages), ref, most)


@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
def test_sequences_that_take_no_part(torch_cuda, shape):  # noqa: F811
    # the first ones, blocks of columns full of them, all of them; what their rows of the table name does not matter
    torch = torch_cuda
    G, D, page, n, heads = shape
    pages = 900 // page + 1
    c = _batch(torch, shape, pages)
    q = c.normal((n, 1, heads * G, D))
    most, lengths, table = _most(c), c.lengths.clone(), c.table.clone()
    for out in (range(1), range(n // 2), range(n - 1), range(n), range(1, n, 2), range(n - 3, n)):
        for s in out:
            c.lengths[s] = (pages * page - 1, 0, page, 1, 3 * page + 7)[s % 5]
            c.table[s, -(-int(c.lengths[s]) // page):] = -5
        _close(c, c.decode_prefix(q), _ref(c, q), most)
        c.lengths.copy_(lengths)
        c.table.copy_(table)


@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
def test_captured_with_everything_changing_between_replays(torch_cuda, shape):  # noqa: F811
    torch = torch_cuda
    G, D, page, n, heads = shape
    pages = 1400 // page + 1
    c = _batch(torch, shape, pages)
    q = c.normal((n, 1, heads * G, D))
    begin, counts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [pages]))
    ws = torch.empty((c.B.sablock_decode_prefix_paged_workspace_bytes(c.pages, 1),), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, NAN, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.B.sablock_decode_prefix_paged(c.pages, q, c.k_pool, c.v_pool, c.table, c.lengths, begin, counts, out, ws)
    table, lengths, most = c.table.clone(), c.lengths.clone(), _most(c)
    for b, m, change in (([0, n], pages, None), ([0, n], pages // 2, "order"), ([2, n - 1], pages - 1, "short"), ([0, n], 1, None), ([0, 0], pages, "short"), ([0, n], pages, None)):
        c.table.copy_(table)
        c.lengths.copy_(lengths)
        if change == "order":                                   # the rows of the prefix in another order of its pages
            c.table[:, : pages // 2] = table[:, torch.randperm(pages // 2, generator=c.gen, device="cuda")]
        if change == "short":
            c.lengths[: n // 2] = torch.arange(n // 2, device="cuda", dtype=torch.int32) * 11
        begin.copy_(torch.tensor(b, dtype=torch.int32))
        counts.fill_(m)
        q.copy_(c.normal(q.shape))
        ws.fill_(0xFF if m % 2 else 0)
        eager = c.decode_prefix(q, b, [m])
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        _close(c, out, _ref(c, q), most)

"""Decode attention that gathers every row's share, against the formula in 64 bits; the attention itself is sablock_decode_paged's, bit for bit."""

import numpy as np
import pytest

from test_gpu_paged import NAN, Cache, torch_cuda  # noqa: F401
from test_gpu_paged_edges import WAYS, _of_way

pytestmark = pytest.mark.gpu

INF = float("inf")


def _weights(c):
    """Gathered so far: some of it large, some that is no number, where a row's new share is all that may be seen."""
    return c.torch.exp(2 * c.torch.randn((c.L, c.n_pages, c.H, c.page), generator=c.gen, device="cuda"))


def _decode(c, q, weights, n_new=1, counts=None, decay=1.0, fill=0xFF):
    torch = c.torch
    ws = torch.full((c.B.sablock_decode_weighed_paged_workspace_bytes(c.pages),), fill, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, NAN, dtype=torch.float32, device="cuda")
    c.B.sablock_decode_weighed_paged(c.pages, q, c.k_pool, c.v_pool, c.table, c.lengths, weights, out, ws, n_new=n_new, decay=decay,
                                     counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    return out


def _shares(c, q, s, l, h):
    """Sum over the query heads of each row's share, in 64 bits."""
    torch, n = c.torch, int(c.lengths[s])
    k = c.rows(c.k_pool, s)[l, h]
    x = q[s, l, h * c.G: (h + 1) * c.G].double().cpu() @ k.T / c.D ** 0.5
    return torch.softmax(x, dim=-1).sum(dim=0) if n else torch.zeros(0, dtype=torch.float64)


def _check(c, q, n_new=1, counts=None, decay=1.0):
    torch = c.torch
    weights = _weights(c)
    was = weights.clone()
    out = _decode(c, q, weights, n_new, counts, decay)
    assert torch.equal(out, c.decode(q))
    got, want, most = weights.double().cpu(), was.double().cpu(), weights.new_zeros(was.shape).double().cpu()
    for s in range(c.n):
        n = int(c.lengths[s])
        fresh = n - min(n_new if counts is None else min(max(counts[s], 0), n_new), n)
        r = torch.arange(n)
        ids = c.table[s].cpu().long()[r // c.page]
        for l in range(c.L):
            for h in range(c.H):
                share = _shares(c, q, s, l, h)
                old = torch.where(r < fresh, decay * want[l, ids, h, r % c.page], 0.0)
                want[l, ids, h, r % c.page] = old + share
                most[l, ids, h, r % c.page] = share
    # A share: fp32 logits of up to 64 in the log2 domain and their distance from the reference, 2^-18 each and as much in the sum, below 2^-16 as in the
    # attention's test; then a product and a sum, half a step of 2^-23 each
    assert bool(((got - want).abs() <= 2.0 ** -16 * most + 2.0 ** -23 * want.abs()).all()), float((got - want).abs().max())
    return weights


@pytest.mark.parametrize("G,D,dtype,page", [(1, 32, "bf16", 16), (2, 64, "bf16", 32), (3, 96, "bf16", 16), (4, 128, "bf16", 16), (4, 128, "bf16", 64), (5, 160, "bf16", 128), (7, 192, "bf16", 16),
                                           (8, 224, "bf16", 256), (16, 128, "bf16", 16), (12, 256, "bf16", 32), (1, 16, "f32", 16), (4, 64, "f32", 64), (7, 80, "f32", 16),
                                           (16, 128, "f32", 32), (5, 240, "f32", 128), (9, 256, "f32", 16)])
@pytest.mark.parametrize("lengths", [[1], [0, 15, 16, 17, 0, 33], [255, 1, 700], [2500], [5, 0, 4097, 31]], ids=str)
def test_groups_heads_pages_and_lengths(torch_cuda, G, D, dtype, page, lengths):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, G * D + lengths[0], lengths, layers=2, heads=2, group=G, D=D, dtype=dtype, page=page, k_axes=(1, 2, 0, 3), pad=16).fill()
    _check(c, c.normal((c.n, 2, 2 * G, D)))


@pytest.mark.parametrize("n_new,counts,decay", [(0, None, 1.0), (1, None, 0.5), (5, None, 1.0), (400, None, 0.9), (30, [30, 0, 7, -3, 100], 0.97), (1, [0, 1, 0, 1, 1], 0.0),
                                                (2 ** 31 - 1, None, 1.0), (3, [2 ** 31 - 1, -2 ** 31, 1, 2, 3], 2.0)], ids=str)
def test_rows_that_have_gathered_nothing_and_decay(torch_cuda, n_new, counts, decay):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 5, [300, 17, 0, 1500, 64], layers=1, heads=2, group=3, D=64).fill()
    q = c.normal((5, 1, 6, 64))
    _check(c, q, n_new, counts, decay)
    # what lies in the rows that have gathered nothing does not matter, nor anywhere if all is forgotten
    took = [min(n_new if counts is None else min(max(counts[s], 0), n_new), n) for s, n in enumerate(c.lengths.tolist())]
    clean = _weights(c)
    dirty = clean.clone()
    for s, n in enumerate(c.lengths.tolist()):
        for r in range(n - took[s] if decay else 0, n):
            dirty[:, int(c.table[s, r // 16]), :, r % 16] = (NAN, INF, -INF)[r % 3]
    _decode(c, q, clean, n_new, counts, decay)
    _decode(c, q, dirty, n_new, counts, decay)
    for s, n in enumerate(c.lengths.tolist()):
        r = torch.arange(n, device="cuda")
        ids = c.table[s].long()[r // 16]
        assert torch.equal(clean[:, ids, :, r % 16], dirty[:, ids, :, r % 16])


@pytest.mark.parametrize("args", [a for a in WAYS if a[8] is None], ids=lambda a: f"{a[0]}-{a[1]}-{a[2]}-{len(a[6])}-{a[7]}")
def test_every_way_of_dealing(torch_cuda, args):  # noqa: F811
    # shares of a sequence sum to the number of its query heads, its rows' weights are nobody else's; the largest problems against the formula
    torch = torch_cuda
    c, _ = _of_way(torch, *args)
    c.k_pool.copy_(c.normal(c.k_pool.shape))
    c.v_pool.copy_(c.normal(c.v_pool.shape))
    q = c.normal((c.n, 1, c.H * c.G, c.D))
    weights = torch.full((1, c.n_pages, c.H, c.page), 7.0, device="cuda")
    out = _decode(c, q, weights, decay=0.0, n_new=0)
    assert torch.equal(out, c.decode(q))
    again = torch.full_like(weights, 7.0)
    _decode(c, q, again, decay=0.0, n_new=0, fill=0x7F)
    assert torch.equal(weights, again)
    left = weights.clone()
    order = np.argsort(-c.lengths.cpu().numpy(), kind="stable")
    for i, s in enumerate(order.tolist()):
        n = int(c.lengths[s])
        r = torch.arange(n, device="cuda")
        ids = c.table[s].long()[r // c.page]
        got = weights[0, ids, :, r % c.page].double()           # row, head
        # every share is off by 2^-16 of itself at most
        assert bool(((got.sum(dim=0) - (c.G if n else 0)).abs() <= 2.0 ** -16 * c.G).all())
        if i < 4:
            for h in range(c.H):
                share = _shares(c, q, s, 0, h)
                assert bool(((got[:, h].cpu() - share).abs() <= 2.0 ** -16 * share).all())
        left[0, ids, :, r % c.page] = 7.0
    assert bool((left == 7.0).all())


def test_pages_that_do_not_exist_and_lengths_beyond_the_table(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 8, [100, 64, 208], heads=2, group=2, D=64).fill()
    c.table = c.table[:, :13].contiguous()
    c.pages = c.B.make_pages(c.k_pool, c.v_pool, c.table, 4)
    q = c.normal((3, 1, 4, 64))
    full = c.table.clone()
    for s, i, at in ((0, 2, -1), (0, 6, c.n_pages), (1, 0, 2 ** 31 - 1), (1, 1, -2 ** 31), (1, 2, -1), (1, 3, c.n_pages)):
        c.table[s, i] = at
    weights = _weights(c)
    was = weights.clone()
    assert torch.equal(_decode(c, q, weights), c.decode(q))
    changed = (weights != was).any(dim=3).any(dim=2)[0]
    reached = {int(full[0, i]) for i in (0, 1, 3, 4, 5)} | {int(x) for x in full[2]}
    assert set(changed.nonzero().flatten().tolist()) == reached
    c.table.copy_(full)
    want = _weights(c)
    got = want.clone()
    # behind a full table the new rows have no place, and the last ones in front of them have gathered before
    some = want.clone()
    _decode(c, q, want, n_new=2, counts=[2, 2, 0])
    c.lengths = torch.tensor([100, 64, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    _decode(c, q, got, n_new=2)
    assert torch.equal(got, want)
    c.lengths = torch.tensor([100, 64, 209], dtype=torch.int32, device="cuda")
    _decode(c, q, some, n_new=2)
    last = int(full[2, 12])
    assert bool((some[0, last, :, 15] != want[0, last, :, 15]).all())
    some[0, last, :, 15] = want[0, last, :, 15]
    assert torch.equal(some, want)
    c.lengths = torch.tensor([-7, 64, 208], dtype=torch.int32, device="cuda")
    again = was.clone()
    assert not _decode(c, q, again)[0].any()
    mine = full[0, :7].long()
    assert torch.equal(again[0, mine], was[0, mine])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [40, 3000])
def test_logits_that_are_infinite_or_no_number(torch_cuda, dtype, rows):  # noqa: F811
    # all logits -infinity: no share, no output; no number: the KV head's weights, and no one else's
    torch = torch_cuda
    c = Cache(torch, 4, [rows, rows], heads=2, group=2, D=64, dtype=dtype).fill()
    q = c.normal((2, 1, 4, 64))
    q[0, 0, 0] = 0.0
    q[0, 0, 0, 0] = -INF
    ids = c.table[0, : -(-rows // 16)].long()
    c.k_pool[0, ids, 0] = c.k_pool[0, ids, 0].abs().clamp(min=0.01)
    c.k_pool[0, ids, 0, :, 1:] = 0.0
    q[0, 0, 1, 0] = 1.0
    q[0, 0, 0, 1:] = 1.0
    weights = torch.zeros((1, c.n_pages, 2, 16), device="cuda")
    out = _decode(c, q, weights)
    assert not out[0, 0, 0].any() and bool(torch.isfinite(out).all())
    r = torch.arange(rows, device="cuda")
    at = c.table[0].long()[r // 16]
    assert bool(((weights[0, at, 0, r % 16].double().sum() - 1).abs() <= 2.0 ** -16))          # the other head's
    c.k_pool[0, int(c.table[1, 1]), 1, 3, 9] = NAN
    _decode(c, q, weights)
    bad = torch.isnan(weights[0])
    r1 = c.table[1].long()[r // 16]
    assert bool(bad[r1, 1, r % 16].all()) and int(bad.sum()) == rows


def test_pools_beyond_two_to_the_31_elements(torch_cuda):  # noqa: F811
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    D, page, n_pages = 32, 16, 2 ** 27 + 2 ** 20
    k_pool, v_pool = (torch.zeros((1, n_pages, 1, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    weights = torch.zeros((1, n_pages, 1, page), device="cuda")                                # 2^31 rows and more
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([40], dtype=torch.int32, device="cuda")
    pages = B.make_pages(k_pool, v_pool, table, 2)
    out = torch.empty((1, 1, 2, D), device="cuda")
    ws = torch.empty((B.sablock_decode_weighed_paged_workspace_bytes(pages),), dtype=torch.uint8, device="cuda")
    q = torch.ones((1, 1, 2, D), dtype=torch.bfloat16, device="cuda")
    B.sablock_decode_weighed_paged(pages, q, k_pool, v_pool, table, lengths, weights, out, ws)
    got = weights[0, table[0].long(), 0].flatten()
    assert bool(((got[:40] - 2 / 40).abs() <= 2.0 ** -20).all()) and not got[40:].any()
    after, len_out, rows_out = torch.tensor([[n_pages - 2, 5, -1]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, 20), dtype=torch.int32, device="cuda")
    weights[0, n_pages - 7, 0, :8] = torch.arange(8, device="cuda").float() + 1
    k_pool[0, n_pages - 7, 0, :8, 0] = torch.arange(8, device="cuda").to(torch.bfloat16) + 1
    ews = torch.empty((B.sablock_evict_paged_workspace_bytes(pages),), dtype=torch.uint8, device="cuda")
    B.sablock_evict_paged(pages, table, lengths, weights, k_pool, v_pool, 20, after, len_out, rows_out, ews, n_first=1, n_last=1)
    assert rows_out[0].tolist() == list(range(12)) + list(range(32, 40)) and len_out.tolist() == [20]
    assert k_pool[0, n_pages - 2, 0, 12:, 0].tolist() == [1, 2, 3, 4] and k_pool[0, 5, 0, :4, 0].tolist() == [5, 6, 7, 8]
    assert weights[0, 5, 0, :4].tolist() == [5, 6, 7, 8]

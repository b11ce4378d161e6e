"""Decode attention of sequences with common pages where the arguments are odd: begins that descend, a workspace for more prefixes."""

import pytest

from test_gpu_paged import NAN, _ref_decode, torch_cuda  # noqa: F401
from test_gpu_paged_prefix import Sharing

pytestmark = pytest.mark.gpu

GUARD = 4096


def _prefix_of(begin, s):
    """The prefix that the kernels look for a sequence in: halves of the begins, whatever their order."""
    lo, hi = 0, len(begin) - 1
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if begin[mid] <= s else (lo, mid)
    return lo


def _guarded(c, q, begin, pages):
    """The call with an output and a workspace that lie between guards, and pools and arguments that stay as they are."""
    torch, B = c.torch, c.B
    b, m = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (begin, pages))
    size = B.sablock_decode_prefix_paged_workspace_bytes(c.pages, len(pages))
    room = torch.full((GUARD + size + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
    line = torch.full((GUARD + q.numel() + GUARD,), NAN, device="cuda")
    out, kept = line[GUARD: GUARD + q.numel()].view(q.shape), [t.clone() for t in (c.k_pool, c.v_pool, c.table, c.lengths, b, m, q)]
    B.sablock_decode_prefix_paged(c.pages, q, c.k_pool, c.v_pool, c.table, c.lengths, b, m, out, room[GUARD: GUARD + size])
    assert bool((room[:GUARD] == 0x5A).all()) and bool((room[GUARD + size:] == 0x5A).all())
    assert bool(torch.isnan(line[:GUARD]).all()) and bool(torch.isnan(line[GUARD + q.numel():]).all())
    for now, was in zip((c.k_pool, c.v_pool, c.table, c.lengths, b, m, q), kept):
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[now.element_size()]
        assert torch.equal(now.contiguous().view(bits), was.contiguous().view(bits))
    return out.clone()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,empty", [(1, 0), (2, 0), (300, 700), (700, 1500)])
def test_begins_that_descend(torch_cuda, pairs, empty, dtype):  # noqa: F811
    # every sequence comes out: with its prefix or, where the pieces of so many have no places, the rows behind it alone, which are many (in pieces) or few
    torch = torch_cuda
    c = Sharing(torch, 3, [(5, 6)], [10, 3000, 0, 4, 900], heads=2, group=2, D=64, dtype=dtype)
    q = c.normal((5, 1, 4, 64))
    begin = [0, 5] * pairs + [0] * empty + ([5] if empty else [0])
    pages = [6] * (len(begin) - 1)
    got = _guarded(c, q, begin, pages).double().cpu()
    whole = _ref_decode(c, q)
    table, lengths = c.table, c.lengths
    c.table, c.lengths = torch.cat([table[:, 6:], table[:, :6]], dim=1), lengths - 96
    behind = _ref_decode(c, q)
    c.table, c.lengths = table, lengths
    most = max(float(c.rows(c.v_pool, s).abs().max()) for s in range(5))
    for s in range(5):
        i = _prefix_of(begin, s)
        member = begin[i] <= s < begin[i + 1]
        # pieces in front of prefix i's, two of each that has sequences (a KV head's, of 96 rows); 512 workgroups' and two heads' two blocks have places
        lost = member and 2 * sum(begin[j] < begin[j + 1] for j in range(i)) + 2 > 512 + 4
        assert lost == (pairs >= 300)
        err = (got[s] - (behind if lost else whole)[s]).abs().max()
        assert err <= 2.0 ** -16 * most, (s, float(err))           # as in the test of the attention without prefixes


def test_as_many_descending_begins_as_a_call_takes_over_long_prefixes(torch_cuda):  # noqa: F811
    # 2 048 times 64 sequences of eight heads behind 2^22 rows: their steps and pieces pass 32 bits.  No pieces of the last prefix have places: V is 1 behind the
    # prefix and 2 in it
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    n, H, G, D, page, m = 64, 8, 4, 128, 256, 2 ** 22 // 256
    c = Sharing(torch, 1, [(2, 1)], [page, 0], heads=H, group=G, D=D, page=page)
    common, behind = int(c.table[0, 0]), int(c.table[0, 1])
    c.k_pool.zero_()
    c.v_pool.fill_(2.0)
    c.v_pool[:, behind] = 1.0
    own = torch.tensor([(s * 5) % 17 for s in range(n)], dtype=torch.int32, device="cuda")
    c.table = torch.full((n, m + 1), common, dtype=torch.int32, device="cuda")
    c.table[:, m] = behind
    c.lengths, c.n = own + m * page, n
    c.pages = B.make_pages(c.k_pool, c.v_pool, c.table, H * G)
    begin = [0, n] * 2047 + [0, 0, n]
    assert len(begin) == 4097 and all(_prefix_of(begin, s) == 4095 for s in range(n))
    q = c.normal((n, 1, H * G, D))
    got = _guarded(c, q, begin, [m] * 4096)
    # equal logits: a share of 1 / rows in each of at most 16 rows, 2^-20 for the quotient and the sum
    assert bool(((got - (own > 0).float()[:, None, None, None]).abs() <= 2.0 ** -20).all())


@pytest.mark.parametrize("D,most", [(128, 64), (128, 5), (256, 40)])
def test_a_cache_serves_calls_with_fewer_prefixes_than_it_has_room_for(torch_cuda, D, most):  # noqa: F811
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    n, H, G, page, m = 64, 2, 4, 16, 20
    cache = B.PagedCache(n, 1, H * G, H, D, page, m + 2 * n, m + 2, torch.bfloat16, "cuda", bounds=False, n_prefixes=most)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D + most)
    for pool in (cache.k_pool, cache.v_pool):
        pool.copy_(torch.randn(pool.shape, generator=gen, device="cuda"))
    cache.page_table[:, :m] = torch.randperm(m, generator=gen, device="cuda").to(torch.int32)
    cache.page_table[:, m:] = m + torch.arange(2 * n, device="cuda", dtype=torch.int32).view(n, 2)
    cache.lengths.copy_(m * page + torch.arange(n, device="cuda") % 33)
    q = torch.randn((n, 1, H * G, D), generator=gen, device="cuda").to(torch.bfloat16)
    want, got = (torch.full(q.shape, NAN, device="cuda") for _ in range(2))
    B.sablock_decode_paged(cache.pages, q, cache.k_pool, cache.v_pool, cache.page_table, cache.lengths, want, cache.ws)
    for prefixes in sorted({1, 2, 3, 4, 7, 8, 31, 40, 64, most}):
        if prefixes > most:
            break
        begin = torch.tensor([n * i // prefixes for i in range(prefixes + 1)], dtype=torch.int32, device="cuda")
        B.sablock_decode_prefix_paged(cache.pages, q, cache.k_pool, cache.v_pool, cache.page_table, cache.lengths, begin,
                                      torch.full((prefixes,), m, dtype=torch.int32, device="cuda"), got.fill_(NAN), cache.prefix_ws)
        # either is off by 2^-16 of the largest value, see the test of the attention without prefixes
        assert bool(((got - want).abs() <= 2 * 2.0 ** -16 * cache.v_pool.abs().max().float()).all()), prefixes

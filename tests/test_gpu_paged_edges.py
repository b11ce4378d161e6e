"""The paged cache's calls where a table, a plan or a type ends, against plain forms in 64 bits."""

import numpy as np
import pytest

from test_gpu_paged import Cache, _ref_append, _ref_decode, _ref_select, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("D,R,interleaved,dtype,page", [(64, 64, False, "bf16", 16), (128, 64, True, "bf16", 64), (96, 96, False, "f32", 32), (40, 0, False, "f32", 16)])
@pytest.mark.parametrize("n_new,beyond,counts", [(1, [0, 1, 2, INT_MAX], None), (1, [-3, 1, 500, 1], [1, 1, 0, 5]), (7, [3, 7, 8, INT_MAX], None), (7, [-2, 3, 6, 200], [7, 2, 0, 7]),
                                                 (64, [1, 40, 64, 90], None), (64, [20, 63, 5, -64], [30, 64, 6, 64])])
def test_append_behind_a_full_table(torch_cuda, D, R, interleaved, dtype, page, n_new, beyond, counts):  # noqa: F811
    # tokens whose rows the table has no room for are dropped: no row in front of them changes, nor its page's bounds; queries are rotated
    torch = torch_cuda
    nl, H, G, cap = 2, 3, 2, 192
    n = len(beyond)
    c = Cache(torch, D + n_new, [cap] * n, layers=nl, heads=H, group=G, D=D, dtype=dtype, page=page)
    c.table = c.table[:, : cap // page].contiguous()            # room for `cap` rows and no more
    c.pages = c.B.make_pages(c.k_pool, c.v_pool, c.table, H * G)
    lengths = [min(cap + x, INT_MAX) for x in beyond]
    took = [n_new if counts is None else min(max(counts[s], 0), n_new) for s in range(n)]
    first = [lengths[s] - took[s] for s in range(n)]
    c.lengths = torch.tensor([min(f, cap) for f in first], dtype=torch.int32, device="cuda")
    c.fill()
    c.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q, k, v = (c.normal((n, nl, h, n_new, D)) for h in (H * G, H, H))
    positions = torch.tensor([131071, 0, 7, 60000], dtype=torch.int32, device="cuda")
    freq = torch.tensor([10000.0 ** (-2 * i / max(R, 1)) for i in range(R // 2)], dtype=torch.float32, device="cuda") if R else None
    q_out = torch.full(q.shape, 77.0, dtype=c.dt, device="cuda")
    want = [t.clone() for t in (c.k_pool, c.v_pool, c.bounds)]
    c.B.sablock_append_paged(c.pages, c.B.make_new_tokens(k, v, q, rotary_dim=R, interleaved=interleaved), k, v, positions if R else None, freq, c.table,
                             c.lengths, c.k_pool, c.v_pool, q=q, q_out=q_out, bounds=c.bounds,
                             counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    (rq, sq), (rk, sk) = _ref_append(c, q, k, took, positions.tolist(), [] if freq is None else freq.tolist(), R, interleaved)
    half = torch.finfo(c.dt).eps / 2

    def close(got, ref, size):                                  # as in the test of appended rows: 2^-21 of |a| + |b|, then half a step of the type
        err = (got.double().cpu() - ref).abs()
        assert bool((err <= half * ref.abs() * (1 + half) + 2.0 ** -21 * size).all()), float(err.max())

    for s in range(n):
        close(q_out[s, :, :, : took[s]], rq[s, :, :, : took[s]], sq[s, :, :, : took[s]])
        assert bool((q_out[s, :, :, took[s]:] == 77.0).all())
        held = max(0, min(took[s], cap - first[s]))             # tokens that the table has room for
        for j in range(held):
            r = first[s] + j
            id, at = int(c.table[s, r // page]), r % page
            close(c.k_pool[:, id, :, at], rk[s, :, :, j], sk[s, :, :, j])
            want[0][:, id, :, at], want[1][:, id, :, at] = c.k_pool[:, id, :, at], v[s, :, :, j]
            rows = c.k_pool[:, id, :, : at + 1].float()
            want[2][:, id, :, 0], want[2][:, id, :, 1] = rows.amin(dim=2).to(c.dt), rows.amax(dim=2).to(c.dt)
    bits = torch.int16 if c.dt == torch.bfloat16 else torch.int32
    for got, ref in zip((c.k_pool, c.v_pool), want):
        assert torch.equal(got.view(bits), ref.view(bits))
    assert torch.equal(torch.nan_to_num(c.bounds.float(), 7.0), torch.nan_to_num(want[2].float(), 7.0))


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (16, "f32")])
@pytest.mark.parametrize("place", [1, 2, 3])
def test_decode_into_any_place_of_an_array(torch_cuda, D, dtype, place):  # noqa: F811
    # an fp32 number's place is enough for the output; a problem of one workgroup, and one in pieces
    torch = torch_cuda
    c = Cache(torch, D, [20, 5000], heads=2, group=3, D=D, dtype=dtype).fill()
    q = c.normal((2, 1, 6, D))
    want = c.decode(q)
    array = torch.full((want.numel() + 8,), 77.0, dtype=torch.float32, device="cuda")
    out = array[place: place + want.numel()].view(want.shape)
    ws = torch.empty((c.B.sablock_decode_paged_workspace_bytes(c.pages),), dtype=torch.uint8, device="cuda")
    c.B.sablock_decode_paged(c.pages, q, c.k_pool, c.v_pool, c.table, c.lengths, out, ws)
    assert torch.equal(out, want) and bool((array[:place] == 77.0).all()) and bool((array[place + want.numel():] == 77.0).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n_new", [1, 70])
def test_append_angles_in_fp32(torch_cuda, interleaved, n_new):  # noqa: F811
    # pairs (1, 0) turn into cosine and sine alone.  Their last rounding: 2^-25 of values below 1; those of the terms behind the first, a tenth of them,
    # a half of that at most
    torch = torch_cuda
    D, n = 128, 4
    c = Cache(torch, 1, [n_new] * n, heads=2, group=1, D=D, dtype="f32")
    one = torch.zeros((n, 1, 2, n_new, D), device="cuda")
    one[..., 0::2] = 1.0 if interleaved else 0.0
    if not interleaved:
        one[..., : D // 2] = 1.0
    positions = torch.tensor([0, 1000, 131072, 2 ** 30], dtype=torch.int32, device="cuda")
    freq = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float32, device="cuda")
    q_out = torch.empty_like(one)
    c.B.sablock_append_paged(c.pages, c.B.make_new_tokens(one, one, one, interleaved=interleaved), one, one, positions, freq, c.table, c.lengths, c.k_pool,
                             c.v_pool, q=one, q_out=q_out)
    angle = (positions.double().cpu()[:, None] + torch.arange(n_new)).numpy()[..., None] * freq.double().cpu().numpy()
    want = np.stack([np.cos(angle), np.sin(angle)], axis=-1 if interleaved else -2).reshape(n, 1, 1, n_new, D)
    got = q_out.double().cpu().numpy()
    assert np.abs(got - want).max() <= 2.0 ** -25 + 2.0 ** -26
    assert torch.equal(c.k_pool[0, c.table[0, 0].long(), :, 0], q_out[0, 0, :, 0])


# ---- the ways of dealing out a decode step -------------------------------------------------------------------------------


def _spread(n, most, least=1):
    """Lengths all over (0, most], the first the longest."""
    return [max(least, int(most * (1 - s * 0.6180339887498949 % 1))) for s in range(n)]


SHORT = [s % 41 for s in range(4096)]
WAYS = [                                                       # way, dtype, D, page, heads, group, lengths, compute units (0: the device's), listed pages
    ("alone", "bf16", 128, 16, 2, 4, [450, 0, 40], 64, None), ("short", "bf16", 128, 16, 2, 4, [510, 0, 40], 64, None),
    ("cut", "bf16", 128, 16, 2, 4, [3000, 10, 1500, 0, 2000], 64, None), ("longer", "bf16", 128, 16, 2, 3, _spread(5, 3000, 1100), 32, None),
    ("even", "bf16", 128, 16, 4, 4, _spread(20, 2600), 4, None), ("even", "bf16", 128, 32, 3, 2, _spread(100, 2300), 16, None),
    ("even", "f32", 64, 64, 3, 7, _spread(33, 5000), 6, None), ("even", "f32", 256, 16, 2, 2, _spread(17, 3000), 8, None), ("even", "bf16", 256, 32, 2, 5, _spread(12, 4000), 8, None),
    ("even", "bf16", 32, 16, 1, 2, [4500 if s % 70 == 3 else n for s, n in enumerate(SHORT)], 8, None),
    ("cut", "bf16", 32, 16, 1, 2, [9000 if s % 400 == 3 else n for s, n in enumerate(SHORT)], 256, None),
    ("even", "bf16", 128, 16, 2, 4, _spread(70, 3000), 4, 80), ("cut", "bf16", 128, 16, 1, 2, _spread(70, 3000), 256, 150), ("even", "f32", 64, 32, 2, 3, _spread(20, 6000), 4, 90),
    ("even", "bf16", 128, 16, 8, 2, _spread(100, 2300), 0, None)]


def _of_way(torch, expected, dtype, D, page, heads, group, lengths, cus, listed):
    from paged_plan import way

    c = Cache(torch, D + len(lengths), lengths, heads=heads, group=group, D=D, dtype=dtype, page=page, k_axes=(0, 2, 1, 3))
    c.pages.compute_units = cus
    real = cus or torch.cuda.get_device_properties(0).multi_processor_count
    assert cus or real == 256
    assert way(dtype, D, page, heads, lengths, c.width, real, listed) == expected
    lst = None if listed is None else torch.randint(-1, c.width, (c.n * heads, listed), generator=c.gen, device="cuda", dtype=torch.int32)
    return c, lst


@pytest.mark.parametrize("args", WAYS, ids=lambda a: f"{a[0]}-{a[1]}-{a[2]}-{len(a[6])}-{a[7]}-{a[8]}")
def test_decode_in_every_way_of_dealing(torch_cuda, args):  # noqa: F811
    torch = torch_cuda
    c, lst = _of_way(torch, *args)
    c.k_pool.copy_(c.normal(c.k_pool.shape))
    c.v_pool.copy_(c.normal(c.v_pool.shape))
    q = c.normal((c.n, 1, c.H * c.G, c.D))
    got, ref = c.decode(q, lst).double().cpu(), _ref_decode(c, q, None if lst is None else lst.cpu())
    assert bool(((got - ref).abs() <= 2.0 ** -16 * 6).all())    # as in the test of many sequences
    assert torch.equal(c.decode(q, lst, ws_fill=0), c.decode(q, lst, ws_fill=0x7F))


@pytest.mark.parametrize("args", [a for a in WAYS if a[8] is None], ids=lambda a: f"{a[0]}-{a[1]}-{a[2]}-{len(a[6])}-{a[7]}")
def test_decode_counts_every_row_once_in_every_way_of_dealing(torch_cuda, args):  # noqa: F811
    # equal logits: the mean of V, which has a one in column r % D of row r.  2^-20 relative as in the test of one sequence
    torch = torch_cuda
    c, _ = _of_way(torch, *args)
    rows = torch.arange(c.width * c.page, device="cuda")
    one = torch.nn.functional.one_hot(rows % c.D, c.D).to(c.dt)
    want = torch.zeros((c.n, c.D), dtype=torch.float64, device="cuda")
    for s, n in enumerate(c.lengths.tolist()):
        if n:
            r = rows[:n]
            ids = c.table[s, r // c.page].long()
            c.k_pool[0, ids, :, r % c.page] = 0.0
            c.v_pool[0, ids, :, r % c.page] = one[:n, None]
            want[s] = torch.bincount(r % c.D, minlength=c.D).double() / n
    got = c.decode(c.normal((c.n, 1, c.H * c.G, c.D))).double()
    assert torch.allclose(got, want[:, None, None].expand_as(got), rtol=2.0 ** -20, atol=0)


# ---- precision -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_probabilities_are_fp32(torch_cuda, dtype):  # noqa: F811
    # Three rows whose logits are exact products.  Column 0 has ones: the shares' sum.  The three parts of a probability are within 2^-26 of it (two would
    # be off by 7e-6 on average), nine products and three terms of the denominator are added, two products and a quotient follow: 14 roundings, 2^-23
    # each where the matrix pipe cuts, below 2^-19.  Columns 1 to 3 have one row's share each: the logit in the log2 domain, at most 1.5,
    # rounds twice, its distance from the reference, at most 12, to 2^-21, the power to 2^-23: 2^-20.7 in a share, twice, and the sum's
    torch = torch_cuda
    n, G, D = 200, 8, 64
    c = Cache(torch, 1, [3] * n, heads=1, group=G, D=D, dtype=dtype)
    at = c.table[:, 0].long()
    first = (torch.rand((n, 3), generator=c.gen, device="cuda") * 2 - 1).to(torch.bfloat16)
    c.k_pool[0, at, 0, :3] = 0.0
    c.k_pool[0, at, 0, :3, 0] = first.to(c.dt)
    c.v_pool[0, at, 0, :3] = 0.0
    c.v_pool[0, at, 0, :3, 0] = 1.0
    for r in range(3):
        c.v_pool[0, at, 0, r, 1 + r] = 1.0
    q = torch.zeros((n, 1, G, D), dtype=c.dt, device="cuda")
    q[..., 0] = torch.arange(1, G + 1, device="cuda").to(c.dt)
    got = c.decode(q)[:, 0].double().cpu()
    share = torch.softmax(first.double().cpu()[:, None] * torch.arange(1, G + 1, dtype=torch.float64)[:, None] / 8, dim=-1)
    assert bool(((got[..., 0] - 1).abs() <= 2.0 ** -19).all()), float((got[..., 0] - 1).abs().max())
    assert bool(((got[..., 1:4] - share).abs() <= (2.0 ** -19.7 + 2.0 ** -19) * share).all())
    assert not got[..., 4:].any()


@pytest.mark.parametrize("D,R,interleaved", [(128, 128, False), (64, 32, True), (96, 96, False)])
@pytest.mark.parametrize("n_new", [1, 45])
def test_append_fp32_rows(torch_cuda, D, R, interleaved, n_new):  # noqa: F811
    # cosine and sine 0.75, the products and their sum one unit of 2^-24 each: 2.75 of |a| + |b|
    torch = torch_cuda
    n = 3
    c = Cache(torch, 2, [n_new + 20] * n, heads=2, group=2, D=D, dtype="f32", page=32)
    q, k, v = (c.normal((n, 1, h, n_new, D)) for h in (4, 2, 2))
    positions = torch.tensor([0, 4000, 131072], dtype=torch.int32, device="cuda")
    freq = torch.tensor([500000.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device="cuda")
    q_out = torch.empty_like(q)
    c.B.sablock_append_paged(c.pages, c.B.make_new_tokens(k, v, q, rotary_dim=R, interleaved=interleaved), k, v, positions, freq, c.table, c.lengths, c.k_pool,
                             c.v_pool, q=q, q_out=q_out)
    (rq, sq), (rk, sk) = _ref_append(c, q, k, [n_new] * n, positions.tolist(), freq.tolist(), R, interleaved)
    assert bool(((q_out.double().cpu() - rq).abs() <= 2.75 * 2.0 ** -24 * sq).all())
    for s in range(n):
        assert bool(((c.rows(c.k_pool, s)[:, :, 20:] - rk[s]).abs() <= 2.75 * 2.0 ** -24 * sk[s]).all())


# ---- lengths that the table does not hold --------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,rows", [("bf16", 224), ("bf16", 3200), ("f32", 3200)])
def test_reads_end_with_the_table(torch_cuda, dtype, rows):  # noqa: F811
    # a length beyond the table counts as all of its rows, a negative one as none: in attention, in attention over listed pages, and in the choice of those
    torch = torch_cuda
    c = Cache(torch, rows, [0, 64, rows], heads=2, group=2, D=64, dtype=dtype)
    c.table = c.table[:, : rows // 16].contiguous()
    c.pages = c.B.make_pages(c.k_pool, c.v_pool, c.table, 4)
    c.fill()
    q = c.normal((3, 1, 4, 64))
    ref, lists = _ref_decode(c, q), _ref_select(c, q, 6, 1, 1)
    listed = _ref_decode(c, q, torch.tensor(lists))
    for over in (rows + 1, rows + 16, INT_MAX):
        c.lengths = torch.tensor([-5, 64, over], dtype=torch.int32, device="cuda")
        assert bool(((c.decode(q).double().cpu() - ref).abs() <= 2.0 ** -16 * 6).all())
        got = c.select(q, 6, 1, 1)
        assert got.tolist() == lists
        assert bool(((c.decode(q, got).double().cpu() - listed).abs() <= 2.0 ** -16 * 6).all())


def test_compress_into_pages_without_dense_buffers(torch_cuda):  # noqa: F811
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B
    from paper_2510_22556_amd import synth

    n, nl, H, D, L, W, budget = 2, 1, 2, 64, 700, 16, 90
    q, k, v = (synth.normal_torch(60 + i, i, (n, nl, h, m, D), "cuda", torch.bfloat16) for i, h, m in ((1, 2 * H, W), (2, H, L), (3, H, L)))
    seg = B.make_segments(np.concatenate([np.arange(0, L - W, 36), [L - W]] * n), np.arange(n + 1) * (-(-(L - W) // 36) + 1), "cuda")
    shape = B.make_shape(q, k, v)
    caches = []
    for dense in (True, False):
        buf = B.Buffers(shape, seg, budget, "cuda", dense=dense)
        cache = B.PagedCache(n, nl, 2 * H, H, D, 16, 20, 8, torch.bfloat16, "cuda")
        cache.page_table.copy_(torch.arange(16, device="cuda").view(n, 8))
        B.compress(shape, q, k, v, seg, [1, 2, 4], budget, buf, cache=cache)
        caches.append(cache)
    assert buf.k_out is None and buf.v_out is None
    for name in ("k_pool", "v_pool", "bounds", "lengths"):
        assert torch.equal(*(getattr(c, name) for c in caches)), name
    with pytest.raises(ValueError, match="cache in pages"):
        B.compress(shape, q, k, v, seg, [1, 2, 4], budget, buf)

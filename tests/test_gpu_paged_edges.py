"""The paged cache's calls where a table, a plan or a type ends, against plain forms in 64 bits."""

import numpy as np
import pytest

from test_gpu_paged import Cache, _ref_append, torch_cuda  # noqa: F401

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

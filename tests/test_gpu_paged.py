"""The paged cache's calls against plain forms in 64 bits: rows into pages, rotated tokens behind them, attention over all pages or over
listed ones, the pages that a score picks; and a run of them together."""

import math

import numpy as np
import pytest

from test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

NAN = float("nan")
GARBAGE = (NAN, float("inf"), float("-inf"), 3e38)


def _dt(torch, name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _garbage(torch, shape, dtype):
    """What memory that nobody has written may hold."""
    n = math.prod(shape)
    return torch.tensor(GARBAGE, device="cuda").to(dtype).repeat(-(-n // 4))[:n].view(shape)


class Cache:
    """Pools full of garbage, a table of scattered pages, and the rows [n_seq, layers, heads, rows, D] that the pages hold."""

    def __init__(self, torch, seed, lengths, layers=1, heads=2, group=2, D=64, dtype="bf16", page=16, spare=2, k_axes=(0, 1, 2, 3), pad=0, capacity=None):
        from paper_2510_22556_amd import binding as B

        self.B, self.torch, self.dt, self.page = B, torch, _dt(torch, dtype), page
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.L, self.H, self.G, self.D, self.n = layers, heads, group, D, len(lengths)
        need = [-(-(c if capacity is None else capacity) // page) for c in lengths]
        self.width, self.n_pages = max(max(need), 1) + 1, sum(need) + spare

        def pool(axes):
            shape = (layers, self.n_pages, heads, page, D)
            inner = [shape[a] for a in axes] + [D + pad]
            t = _garbage(torch, inner, self.dt)[..., :D]
            return t.permute([axes.index(a) for a in range(4)] + [4])

        self.k_pool, self.v_pool = pool(list(k_axes)), pool([0, 1, 2, 3])
        perm = torch.randperm(self.n_pages, generator=self.gen, device="cuda").to(torch.int32)
        self.table = torch.full((self.n, self.width), -7, dtype=torch.int32, device="cuda")
        at = 0
        for s, m in enumerate(need):
            self.table[s, :m] = perm[at: at + m]
            at += m
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.bounds = _garbage(torch, (layers, self.n_pages, heads, 2, D), self.dt)
        self.pages = B.make_pages(self.k_pool, self.v_pool, self.table, heads * group)

    def normal(self, shape, dtype=None):
        return self.torch.randn(shape, generator=self.gen, device="cuda", dtype=self.torch.float32).to(dtype or self.dt)

    def fill(self, scale=1.0):
        """Random rows into the pages and their bounds; the rest keeps its garbage."""
        torch = self.torch
        for s, rows in enumerate(self.lengths.tolist()):
            for i in range(-(-rows // self.page)):
                n, id = min(self.page, rows - i * self.page), int(self.table[s, i])
                offset = self.normal((1, self.H, 1, self.D), torch.float32)
                self.k_pool[:, id, :, :n] = (self.normal((self.L, self.H, n, self.D), torch.float32) * scale + offset[0] * 0.5).to(self.dt)
                self.v_pool[:, id, :, :n] = self.normal((self.L, self.H, n, self.D))
                self.bounds[:, id, :, 0] = self.k_pool[:, id, :, :n].float().amin(dim=2).to(self.dt)
                self.bounds[:, id, :, 1] = self.k_pool[:, id, :, :n].float().amax(dim=2).to(self.dt)
        return self

    def rows(self, pool, s, n=None):
        """[layers, heads, rows, D] of sequence s in 64 bits on the host."""
        n = int(self.lengths[s]) if n is None else n
        ids = self.table[s, : -(-n // self.page)].long()
        return pool[:, ids].permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :n].double().cpu()

    def decode(self, q, page_list=None, ws_fill=0xFF, **kw):
        ws = self.torch.full((self.B.sablock_decode_paged_workspace_bytes(self.pages),), ws_fill, dtype=self.torch.uint8, device="cuda")
        out = self.torch.full(q.shape, NAN, dtype=self.torch.float32, device="cuda")
        self.B.sablock_decode_paged(self.pages, q, self.k_pool, self.v_pool, self.table, self.lengths, out, ws, page_list=page_list, **kw)
        return out

    def select(self, q, pick, first=1, last=1):
        ws = self.torch.full((self.B.sablock_select_pages_workspace_bytes(self.pages),), 0xFF, dtype=self.torch.uint8, device="cuda")
        out = self.torch.full((self.n * self.L * self.H, pick), -99, dtype=self.torch.int32, device="cuda")
        self.B.sablock_select_pages(self.pages, q, self.bounds, self.table, self.lengths, pick, out, ws, n_first=first, n_last=last)
        return out


def _attention(torch, q, k, v):
    """q [G, D], k, v [rows, D] in 64 bits: one query per head; zeros without rows."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    return torch.softmax(q @ k.T / math.sqrt(q.shape[1]), dim=-1) @ v


def _ref_decode(c, q, page_list=None):
    torch = c.torch
    out = torch.zeros(q.shape, dtype=torch.float64)
    qh = q.double().cpu()
    for s in range(c.n):
        n = int(c.lengths[s])
        k, v = c.rows(c.k_pool, s), c.rows(c.v_pool, s)
        for l in range(c.L):
            for h in range(c.H):
                at = torch.arange(n)
                if page_list is not None:
                    p = (s * c.L + l) * c.H + h
                    entries = page_list[p, : -(-n // c.page)].tolist()
                    at = torch.tensor([r for e in entries if 0 <= e < -(-n // c.page) for r in range(e * c.page, min(n, (e + 1) * c.page))], dtype=torch.long)
                out[s, l, h * c.G: (h + 1) * c.G] = _attention(torch, qh[s, l, h * c.G: (h + 1) * c.G], k[l, h][at], v[l, h][at])
    return out


def _check_decode(c, q, page_list=None):
    # fp32 logits of up to 64 in the log2 domain: half a unit of 2^-17 in the last place and as much again in the sum and the
    # exponential, 2^-17 in a share; shares of values of both signs: twice that of the largest value
    got = c.decode(q, page_list).double().cpu()
    most = max(float(c.rows(c.v_pool, s).abs().max()) if int(c.lengths[s]) > 0 else 0.0 for s in range(c.n))
    ref = _ref_decode(c, q, page_list)
    err = (got - ref).abs().max()
    assert err <= 2.0 ** -16 * max(most, 1.0), float(err)


# ---- rows into pages -----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("D,dtype,page", [(8, "f32", 16), (64, "bf16", 16), (96, "bf16", 32), (128, "bf16", 64), (256, "bf16", 256), (256, "f32", 16), (40, "bf16", 128)])
@pytest.mark.parametrize("L,W,budget,window", [(70, 8, 20, True), (300, 16, 283, True), (300, 16, 1000, True), (50, 1, 49, False), (40, 33, 0, True), (40, 33, 0, False)])
def test_compact_into_pages(torch_cuda, D, dtype, page, L, W, budget, window):  # noqa: F811
    torch = torch_cuda
    T, n, nl, H = L - W, 2, 2, 3
    kept = min(budget, T)
    rows = kept + (W if window else 0)
    c = Cache(torch, L + D, [rows] * n, layers=nl, heads=H, D=D, dtype=dtype, page=page, k_axes=(1, 0, 3, 2), pad=8)
    B = c.B
    k, v = (c.normal((n, nl, H, L, D)) for _ in range(2))
    k[0, 0, 0, 3, :4] = torch.tensor([0.0, -0.0, 1e30, -1e30], device="cuda").to(c.dt)
    idx = torch.full((n * nl * H, max(budget, 1)), -1, dtype=torch.int32, device="cuda")
    for p in range(n * nl * H):
        idx[p, :kept] = torch.randperm(T, generator=c.gen, device="cuda")[:kept].sort().values.to(torch.int32)
    if kept > 2:
        idx[1, 1], idx[2, 0] = L + 5, -3                        # entries that name no token: rows of zeros
        idx[3, 2] = idx[3, 1]                                   # the same token twice
    shape = B.make_shape(torch.zeros((n, nl, H, W, D), dtype=c.dt, device="cuda"), k, v)
    before = [t.clone() for t in (c.k_pool, c.v_pool, c.bounds)]
    got_len = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    B.sablock_compact_paged(shape, k, v, idx, budget, window, c.pages, c.table, c.k_pool, c.v_pool, bounds=c.bounds, lengths_out=got_len)
    assert got_len.tolist() == [rows] * n
    want_k, want_v, want_b = before
    for s in range(n):
        for l in range(nl):
            for h in range(H):
                at = idx[(s * nl + l) * H + h, :kept].long()
                at = torch.cat([at, torch.arange(T, T + (W if window else 0), device="cuda")])
                ok = ((at >= 0) & (at < L))[:, None]
                for src, want in ((k, want_k), (v, want_v)):
                    r = torch.where(ok, src[s, l, h, at.clamp(0, L - 1)], torch.zeros((), dtype=c.dt, device="cuda"))
                    for i in range(-(-rows // page)):
                        part, id = r[i * page: (i + 1) * page], int(c.table[s, i])
                        want[l, id, h, : part.shape[0]] = part
                        if src is k:
                            want_b[l, id, h, 0], want_b[l, id, h, 1] = part.float().amin(dim=0).to(c.dt), part.float().amax(dim=0).to(c.dt)
    bits = torch.int16 if c.dt == torch.bfloat16 else torch.int32
    for got, want in ((c.k_pool, want_k), (c.v_pool, want_v)):
        assert torch.equal(got.contiguous().view(bits), want.contiguous().view(bits))          # garbage that is not theirs too
    assert torch.equal(torch.nan_to_num(c.bounds.float(), 7.0), torch.nan_to_num(want_b.float(), 7.0))


def test_compact_drops_rows_of_pages_that_do_not_exist(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 5, [60, 60], heads=2, D=64)
    c.table[0, 1], c.table[1, 0] = c.n_pages, -1
    k, v = (c.normal((2, 1, 2, 100, 64)) for _ in range(2))
    idx = torch.arange(52, dtype=torch.int32, device="cuda").repeat(4, 1)
    shape = c.B.make_shape(torch.zeros((2, 1, 2, 8, 64), dtype=c.dt, device="cuda"), k, v)
    before = c.k_pool.clone()
    c.B.sablock_compact_paged(shape, k, v, idx, 52, True, c.pages, c.table, c.k_pool, c.v_pool)
    written = {int(x) for x in (c.table[0, 0], *c.table[0, 2:4], *c.table[1, 1:4])}
    for id in range(c.n_pages):
        same = torch.equal(c.k_pool[:, id].view(torch.int16), before[:, id].view(torch.int16))
        assert same == (id not in written)
    assert torch.equal(c.k_pool[0, int(c.table[0, 0])], k[0, 0, :, :16]) and torch.equal(c.k_pool[0, int(c.table[1, 3]), :, 4:12], k[1, 0, :, 92:])


# ---- new tokens ----------------------------------------------------------------------------------------------------------


def _ref_append(c, q, k, counts, positions, freq, R, interleaved):
    """Rotated q and k in 64 bits and |a| + |b| of every pair."""
    torch = c.torch
    res = []
    for x in (q, k):
        x = x.double().cpu().clone()
        size = x.abs()
        for s in range(c.n):
            at = torch.arange(x.shape[3], dtype=torch.float64) + int(positions[s])
            for i in range(R // 2):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
                t = at * float(freq[i])
                u, w = x[s, :, :, :, a].clone(), x[s, :, :, :, b].clone()
                x[s, :, :, :, a], x[s, :, :, :, b] = u * torch.cos(t) - w * torch.sin(t), w * torch.cos(t) + u * torch.sin(t)
                size[s, :, :, :, a] = size[s, :, :, :, b] = u.abs() + w.abs()
        res.append((x, size))
    return res


@pytest.mark.parametrize("D,R,interleaved,dtype,page", [(64, 64, False, "bf16", 16), (128, 128, False, "bf16", 64), (128, 64, True, "bf16", 32), (96, 96, True, "f32", 16),
                                                       (256, 256, False, "f32", 256), (256, 256, False, "bf16", 128), (40, 16, False, "f32", 16),
                                                       (72, 0, False, "bf16", 32), (8, 0, False, "f32", 16)])
@pytest.mark.parametrize("n_new,lengths,counts", [(1, [1, 16, 17, 1000], None), (1, [5, 40, 0, 33], [1, 0, 1, -4]), (7, [7, 20, 64, 257], [7, 3, 7, 0]),
                                                  (130, [130, 400, 500, 131], None), (130, [1, 299, 300, 131], [130, 77, 300, 1])])
def test_append(torch_cuda, D, R, interleaved, dtype, page, n_new, lengths, counts):  # noqa: F811
    torch = torch_cuda
    nl, H, G = 2, 3, 2
    c = Cache(torch, D + R + n_new, lengths, layers=nl, heads=H, group=G, D=D, dtype=dtype, page=page, k_axes=(1, 3, 0, 2))
    B, n = c.B, c.n
    took = [min(n_new if counts is None else min(max(counts[s], 0), n_new), lengths[s]) for s in range(n)]
    before = c.lengths - torch.tensor(took, dtype=torch.int32, device="cuda")
    c.lengths, after = before, c.lengths
    c.fill()
    c.lengths = after
    qkv = c.normal((n, n_new, nl, H * (G + 2), D)).permute(0, 2, 3, 1, 4)
    q, k, v = qkv[:, :, : H * G], qkv[:, :, H * G: H * (G + 1)], qkv[:, :, H * (G + 1):]
    positions = torch.tensor([131071, 0, 7, 2 ** 30], dtype=torch.int32, device="cuda")
    freq = torch.tensor([10000.0 ** (-2 * i / max(R, 1)) for i in range(R // 2)], dtype=torch.float32, device="cuda") if R else None
    q_out = torch.full((n, nl, H * G, n_new, D), 77.0, dtype=c.dt, device="cuda")
    tokens = B.make_new_tokens(k, v, q, rotary_dim=R, interleaved=interleaved)
    old = [t.clone() for t in (c.k_pool, c.v_pool, c.bounds)]
    B.sablock_append_paged(c.pages, tokens, k, v, positions if R else None, freq, c.table, c.lengths, c.k_pool, c.v_pool, q=q, q_out=q_out,
                           counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"), bounds=c.bounds)
    (rq, sq), (rk, sk) = _ref_append(c, q, k, took, positions.tolist(), [] if freq is None else freq.tolist(), R, interleaved)
    # the angle's fraction of a turn in fp32: 2^-25 of half a turn, pi 2^-25 in the angle; sine and cosine 2 units of 2^-24; two
    # products and their sum 2^-24 each: 2^-21 of |a| + |b| covers them.  Then half a step of the type.
    half = torch.finfo(c.dt).eps / 2

    def close(got, ref, size, exact_from):
        err = (got.double().cpu() - ref).abs()
        assert bool((err <= half * ref.abs() * (1 + half) + 2.0 ** -21 * size).all()), float(err.max())
        assert bool((err[..., exact_from:] == 0).all())

    live = torch.zeros((n, n_new), dtype=torch.bool)
    for s in range(n):
        live[s, : took[s]] = True
        close(q_out[s, :, :, : took[s]], rq[s, :, :, : took[s]], sq[s, :, :, : took[s]], R)
        assert bool((q_out[s, :, :, took[s]:] == 77.0).all())
        a, b = lengths[s] - took[s], lengths[s]
        if took[s]:
            close(c.rows(c.k_pool, s)[:, :, a:b], rk[s, :, :, : took[s]], sk[s, :, :, : took[s]], R)
            assert torch.equal(c.rows(c.v_pool, s)[:, :, a:b], v[s, :, :, : took[s]].double().cpu())
        # the bounds are those of the rows that the pages now hold, untouched pages' and all other memory as before
        for i in range(a // page, -(-b // page) if took[s] else 0):
            id, m = int(c.table[s, i]), min(page, b - i * page)
            held = c.k_pool[:, id, :, :m].float()
            assert torch.equal(c.bounds[:, id, :, 0].float(), held.amin(dim=2)) and torch.equal(c.bounds[:, id, :, 1].float(), held.amax(dim=2))
            f = max(a - i * page, 0)
            for pool, was in ((c.k_pool, old[0]), (c.v_pool, old[1])):
                was[:, id, :, f:m] = pool[:, id, :, f:m]
            old[2][:, id] = c.bounds[:, id]
    bits = torch.int16 if c.dt == torch.bfloat16 else torch.int32
    for got, want in zip((c.k_pool, c.v_pool, c.bounds), old):
        assert torch.equal(got.contiguous().view(bits), want.contiguous().view(bits))


def test_append_without_queries_bounds_or_pages(torch_cuda):  # noqa: F811
    # a page that does not exist takes nothing, the others their rows; the token's position does not depend on its row
    torch = torch_cuda
    c = Cache(torch, 3, [40, 40], D=64)
    c.table[0, 2] = 2 ** 31 - 1
    k, v = (c.normal((2, 1, 2, 12, 64)) for _ in range(2))
    tokens = c.B.make_new_tokens(k, v, rotary_dim=0)
    before = c.k_pool.clone()
    c.B.sablock_append_paged(c.pages, tokens, k, v, None, None, c.table, c.lengths, c.k_pool, c.v_pool)
    for id in range(c.n_pages):
        changed = not torch.equal(c.k_pool[:, id].view(torch.int16), before[:, id].view(torch.int16))
        assert changed == (id in (int(c.table[0, 1]), int(c.table[1, 1]), int(c.table[1, 2])))
    assert torch.equal(c.k_pool[0, int(c.table[0, 1]), :, 12:], k[0, 0, :, :4]) and torch.equal(c.v_pool[0, int(c.table[1, 2]), :, :8], v[1, 0, :, 4:])


# ---- attention -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("G,D,dtype,page", [(1, 32, "bf16", 16), (2, 64, "bf16", 32), (3, 96, "bf16", 16), (4, 128, "bf16", 16), (4, 128, "bf16", 64), (5, 160, "bf16", 128), (7, 192, "bf16", 16),
                                           (8, 224, "bf16", 256), (16, 128, "bf16", 16), (12, 256, "bf16", 32), (1, 16, "f32", 16), (4, 64, "f32", 64), (7, 80, "f32", 16),
                                           (16, 128, "f32", 32), (5, 240, "f32", 128), (9, 256, "f32", 16)])
@pytest.mark.parametrize("lengths", [[1], [0, 15, 16, 17, 0, 33], [255, 1, 700], [2500], [5, 0, 4097, 31]], ids=str)
def test_decode_groups_heads_pages_and_lengths(torch_cuda, G, D, dtype, page, lengths):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, G * D + lengths[0], lengths, layers=2, heads=2, group=G, D=D, dtype=dtype, page=page, k_axes=(1, 2, 0, 3), pad=16).fill()
    _check_decode(c, c.normal((c.n, 2, 2 * G, D)))


@pytest.mark.parametrize("D,dtype,page,n,most", [(128, "bf16", 16, 150, 90), (128, "bf16", 32, 150, 1500), (64, "f32", 16, 70, 900), (256, "bf16", 16, 300, 700), (32, "bf16", 16, 4096, 40)])
def test_decode_many_sequences(torch_cuda, D, dtype, page, n, most):  # noqa: F811
    # more sequences than lanes, empty ones among them, first and last; most short, some longer than a workgroup takes alone
    torch = torch_cuda
    rng = np.random.default_rng(n + most)
    lengths = [0 if rng.random() < 0.15 else int(rng.integers(1, most if rng.random() < 0.2 else 50)) for _ in range(n)]
    lengths[0] = lengths[-1] = 0
    lengths[n // 2] = 5 * most
    c = Cache(torch, n, lengths, heads=1 if n > 1000 else 3, group=2, D=D, dtype=dtype, page=page, k_axes=(0, 2, 1, 3))
    # one fill for all pages: the rows behind the sequences' ends are then ordinary numbers, garbage is the other tests'
    c.k_pool.copy_(c.normal(c.k_pool.shape))
    c.v_pool.copy_(c.normal(c.v_pool.shape))
    q = c.normal((n, 1, 2 * c.H, D))
    got, ref = c.decode(q).double().cpu(), _ref_decode(c, q)
    assert bool(((got - ref).abs() <= 2.0 ** -16 * 6).all())
    lst = torch.randint(0, 12, (n * c.H, 6), generator=c.gen, device="cuda", dtype=torch.int32)
    got, ref = c.decode(q, lst).double().cpu(), _ref_decode(c, q, lst.cpu())
    assert bool(((got - ref).abs() <= 2.0 ** -16 * 6).all())


def test_decode_tables_for_more_steps_than_32_bits_count(torch_cuda):  # noqa: F811
    # 40 sequences with room for 2^30 rows each: their steps are summed in 64 bits
    torch = torch_cuda
    c = Cache(torch, 3, [3000 if s % 7 == 3 else s * 11 for s in range(40)], heads=1, group=2, D=16, dtype="f32", page=256).fill()
    q = c.normal((40, 1, 2, 16))
    ref = _ref_decode(c, q)
    wide = torch.full((40, 1 << 22), -1, dtype=torch.int32, device="cuda")
    wide[:, : c.width] = c.table
    c.table, c.pages = wide, c.B.make_pages(c.k_pool, c.v_pool, wide, 2)
    assert bool(((c.decode(q).double().cpu() - ref).abs() <= 2.0 ** -16 * 6).all())


@pytest.mark.parametrize("G,D,dtype,page", [(4, 128, "bf16", 16), (7, 64, "bf16", 128), (16, 256, "bf16", 32), (3, 64, "f32", 16), (8, 256, "f32", 64)])
def test_decode_counts_every_row_once(torch_cuda, G, D, dtype, page):  # noqa: F811
    # equal logits: the mean of V.  V[r] = 1 in column r % D and 0 elsewhere, so a row that is lost, comes twice, or is not the
    # sequence's shows as a share of 1 / length; 2^-20 relative for the quotient and the sums of whole numbers
    torch = torch_cuda
    for n in (1, 17, 63, 64, 65, 1000, 3001, 16 * 129 + 1):
        c = Cache(torch, n, [n, max(n - 1, 1)], heads=1, group=G, D=D, dtype=dtype, page=page).fill()
        for s, rows in enumerate(c.lengths.tolist()):
            r = torch.arange(rows, device="cuda")
            ids = c.table[s, r // page].long()
            c.k_pool[0, ids, 0, r % page] = 0.0
            one = torch.nn.functional.one_hot(r % D, D).to(c.dt)
            c.v_pool[0, ids, 0, r % page] = one
            want = one.double().mean(dim=0)
            got = c.decode(c.normal((2, 1, G, D)))[s, 0].double()
            assert torch.allclose(got, want.expand_as(got), rtol=2.0 ** -20, atol=0), (n, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("late,scale", [(5.0, 2.0 ** 108), (200.0, 2.0 ** 108), (41.0, 2.0 ** -100), (-300.0, 1.0)])
def test_decode_logits_that_rise_late_and_values_near_the_ends(torch_cuda, dtype, late, scale):  # noqa: F811
    torch = torch_cuda
    D, rows = 64, 3000
    c = Cache(torch, 9, [rows, 40], heads=1, group=3, D=D, dtype=dtype).fill()
    for s, m in enumerate((rows, 40)):
        r = torch.arange(m, device="cuda")
        ids = c.table[s, r // 16].long()
        c.k_pool[0, ids, 0, r % 16] = torch.nn.functional.one_hot(torch.zeros_like(r), D).to(c.dt) * (r >= m // 2).to(c.dt)[:, None] * late
        c.v_pool[0, ids, 0, r % 16] = (c.v_pool[0, ids, 0, r % 16].float() * scale).to(c.dt)
    q = torch.zeros((2, 1, 3, D), device="cuda")
    q[..., 0] = D ** 0.5
    got, ref = c.decode(q.to(c.dt)).double().cpu(), _ref_decode(c, q.to(c.dt))
    most = max(float(c.rows(c.v_pool, s).abs().max()) for s in range(2))
    assert bool(((got - ref).abs() <= 2.0 ** -15 * most).all())         # logits up to 2^8.8 in the log2 domain: 2^-16 in a share


def test_append_of_more_heads_than_a_grid_has_places(torch_cuda):  # noqa: F811
    # one token of 60 000 KV heads and 960 000 query heads
    torch = torch_cuda
    c = Cache(torch, 4, [3], heads=60000, group=16, D=8, dtype="f32")
    k, v, q = c.normal((1, 1, 60000, 1, 8)), c.normal((1, 1, 60000, 1, 8)), c.normal((1, 1, 960000, 1, 8))
    q_out = torch.empty_like(q)
    c.B.sablock_append_paged(c.pages, c.B.make_new_tokens(k, v, q, rotary_dim=0), k, v, None, None, c.table, c.lengths, c.k_pool, c.v_pool, q=q, q_out=q_out)
    at = int(c.table[0, 0])
    assert torch.equal(q_out, q) and torch.equal(c.k_pool[0, at, :, 2], k[0, 0, :, 0]) and torch.equal(c.v_pool[0, at, :, 2], v[0, 0, :, 0])


@pytest.mark.parametrize("dtype,at", [("bf16", 0), ("bf16", 99), ("f32", 50)])
def test_decode_a_row_that_is_not_a_number_stays_with_its_head(torch_cuda, dtype, at):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 4, [100, 100], heads=2, group=2, D=64, dtype=dtype).fill()
    q = c.normal((2, 1, 4, 64))
    clean = c.decode(q)
    c.k_pool[0, int(c.table[1, at // 16]), 1, at % 16, 5] = NAN
    got = c.decode(q)
    assert bool(torch.isnan(got[1, 0, 2:]).all())
    got[1, 0, 2:] = clean[1, 0, 2:]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [20, 3000])
def test_decode_an_infinite_value_stays_infinite(torch_cuda, dtype, rows):  # noqa: F811
    # in its column, for every head; also where the row's probability is a power of two, whose lower bits are zeros
    torch = torch_cuda
    c = Cache(torch, 4, [rows, rows], heads=2, group=3, D=64, dtype=dtype).fill()
    q = c.normal((2, 1, 6, 64))
    q[0, 0, 1] = 0.0
    clean = c.decode(q)
    c.v_pool[0, int(c.table[0, 0]), 0, 7, 3], c.v_pool[0, int(c.table[0, 1]), 0, 1, 60] = float("inf"), float("-inf")
    got = c.decode(q)
    assert bool((got[0, 0, :3, 3] == float("inf")).all()) and bool((got[0, 0, :3, 60] == float("-inf")).all())
    got[0, 0, :3, 3], got[0, 0, :3, 60] = clean[0, 0, :3, 3], clean[0, 0, :3, 60]
    assert torch.equal(got, clean)


def test_decode_skips_pages_that_do_not_exist_and_bounds_lengths(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 8, [100, 64, 200], heads=2, group=2, D=64).fill()
    q = c.normal((3, 1, 4, 64))
    for s, i, id in ((0, 2, -1), (0, 6, c.n_pages), (1, 0, 2 ** 31 - 1), (1, 1, -2 ** 31), (1, 2, -1), (1, 3, c.n_pages)):
        c.table[s, i] = id
    got = c.decode(q).double().cpu()
    assert not got[1].any()                                     # no page: no row
    keep = torch.tensor([r for r in range(100) if r // 16 not in (2, 6)])
    safe = c.table.clone()
    c.table = c.table.clamp(0, c.n_pages - 1)
    k, v = c.rows(c.k_pool, 0)[0][:, keep], c.rows(c.v_pool, 0)[0][:, keep]
    c.table = safe
    for h in range(2):
        ref = _attention(torch, q[0, 0, 2 * h: 2 * h + 2].double().cpu(), k[h], v[h])
        assert bool(((got[0, 0, 2 * h: 2 * h + 2] - ref).abs() <= 2.0 ** -16 * 5).all())
    ok = Cache(torch, 8, [100, 64, 200], heads=2, group=2, D=64).fill()
    want = ok.decode(q)
    ok.lengths = torch.tensor([-5, 64, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ok.table[2, 12] = ok.table[2, 11]                           # 200 rows end in page 12, the table in page 13: a length beyond it ends there
    got = ok.decode(q)
    assert not got[0].any() and torch.equal(got[1], want[1])


@pytest.mark.parametrize("G,D,dtype,page", [(4, 128, "bf16", 16), (7, 64, "bf16", 64), (3, 96, "f32", 32)])
def test_decode_over_listed_pages(torch_cuda, G, D, dtype, page):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 6, [1000, 3, 0, 2000, 65], layers=2, heads=2, group=G, D=D, dtype=dtype, page=page).fill()
    q, P = c.normal((5, 2, 2 * G, D)), 5 * 2 * 2
    for width in (1, 5, 70):
        lst = torch.full((P, width), -1, dtype=torch.int32)
        rng = np.random.default_rng(width)
        for p in range(P):
            n = -(-int(c.lengths[p // 4]) // page)
            m = min(n, width)
            if m:
                lst[p, :m] = torch.as_tensor(rng.permutation(n)[:m].astype(np.int32))
        if width == 5:
            lst[0, 1], lst[1, 2], lst[2, 0] = -1, 10 ** 6, 2 ** 31 - 1          # name no page of the sequence
            lst[3, 1] = lst[3, 0]                               # twice
            lst[4:8, 1:] = 0                                    # behind the entries that a sequence of one page has: not read
        _check_decode(c, q, lst.cuda())


def test_decode_lists_of_all_pages_are_the_whole(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 6, [777, 40], heads=2, group=4, D=128).fill()
    q = c.normal((2, 1, 8, 128))
    lst = torch.arange(c.width, dtype=torch.int32, device="cuda").repeat(4, 1)
    a, b = c.decode(q), c.decode(q, lst)
    assert bool(((a - b).abs() <= 2.0 ** -16 * 5).all())


# ---- the pages that a score picks ----------------------------------------------------------------------------------------


def _ref_select(c, q, pick, first, last):
    torch = c.torch
    lists = []
    qh, b = q.double().cpu(), c.bounds.double().cpu()
    for s in range(c.n):
        n = -(-int(c.lengths[s]) // c.page)
        ids = c.table[s, :n].long().cpu()
        for l in range(c.L):
            for h in range(c.H):
                lo, hi = b[l, ids, h, 0], b[l, ids, h, 1]
                x = qh[s, l, h * c.G: (h + 1) * c.G]
                score = torch.maximum(x[:, None] * lo, x[:, None] * hi).sum(dim=-1).amax(dim=0).float().tolist()
                forced = set(range(min(first, n))) | set(range(max(0, n - last), n))
                if n <= pick:
                    got = list(range(n))
                else:
                    rest = sorted((i for i in range(n) if i not in forced), key=lambda i: (-score[i], i))
                    got = sorted(list(forced) + rest[: pick - len(forced)])
                lists.append(got + [-1] * (pick - len(got)))
    return lists


@pytest.mark.parametrize("G,D,dtype,page", [(1, 32, "bf16", 16), (4, 128, "bf16", 16), (7, 96, "bf16", 32), (8, 256, "bf16", 16), (16, 64, "bf16", 16), (4, 128, "f32", 16),
                                           (5, 40, "f32", 16), (9, 256, "f32", 16), (3, 8, "bf16", 16), (2, 88, "bf16", 16),
                                             (16, 16, "f32", 16), (12, 224, "bf16", 64), (6, 128, "bf16", 32), (13, 32, "f32", 16), (7, 200, "f32", 16)])
@pytest.mark.parametrize("pick,first,last", [(1, 0, 0), (1, 0, 1), (8, 1, 1), (64, 2, 3), (300, 0, 1)])
def test_select(torch_cuda, G, D, dtype, page, pick, first, last):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, G + D + pick, [0, 5, 8 * page, 8 * page + 1, 100 * page - 3], layers=2, heads=2, group=G, D=D, dtype=dtype, page=page).fill()
    q = c.normal((5, 2, 2 * G, D))
    assert c.select(q, pick, first, last).tolist() == _ref_select(c, q, pick, first, last)


def test_select_of_equal_scores_and_of_what_is_no_number(torch_cuda):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 2, [16 * 2000], heads=1, group=2, D=32)
    q = torch.ones((1, 1, 2, 32), dtype=c.dt, device="cuda")
    c.bounds.zero_()
    assert c.select(q, 40, 1, 2)[0].tolist() == list(range(38)) + [1998, 1999]
    order = c.table[0, :2000].long()
    c.bounds[0, order[700], 0] = 1.0                            # the best, then two of the same
    c.bounds[0, order[1500], 0], c.bounds[0, order[900], 0] = 0.5, 0.5
    assert c.select(q, 5, 0, 1)[0].tolist() == [0, 700, 900, 1500, 1999]
    assert c.select(q, 3, 0, 1)[0].tolist() == [700, 900, 1999]
    c.bounds[0, order[1200], 0, 1, 3] = NAN
    assert c.select(q, 2, 0, 1)[0].tolist() == [1200, 1999]
    c.table[0, 700] = -1                                        # no page: below every number
    assert c.select(q, 3, 0, 0)[0].tolist() == [900, 1200, 1500]
    c.bounds.fill_(-1.0)
    assert c.select(q, 1999, 0, 0)[0].tolist() == [i for i in range(2000) if i != 700]


@pytest.mark.parametrize("G,D,dtype", [(3, 64, "bf16"), (16, 96, "bf16"), (5, 128, "f32")])
def test_select_with_infinite_bounds(torch_cuda, G, D, dtype):  # noqa: F811
    # infinite, or no number, by the side that the query takes; one page's stay with it, and one head's
    torch = torch_cuda
    inf = float("inf")
    c = Cache(torch, D, [16 * 200, 16 * 200], heads=2, group=G, D=D, dtype=dtype).fill()
    q = c.normal((2, 1, 2 * G, D))
    plain = _ref_select(c, q, 20, 1, 1)
    assert c.select(q, 20, 1, 1).tolist() == plain
    q[..., 5], q[..., 6] = 1.0, -1.0
    order = c.table[0, :200].long()
    for page, e, side, value in ((50, 5, 1, inf), (60, 5, 0, -inf), (70, 6, 0, -inf), (80, 6, 1, inf)):      # inf, NaN, inf, NaN
        c.bounds[0, order[page], 0, side, e] = value
    c.bounds[0, order[90], 0, 1, 5] = -inf                                                                   # below all
    c.bounds[0, order[90], 0, 0, 5] = -1.0
    got = c.select(q, 4, 0, 0)
    assert got[0].tolist() == [50, 60, 70, 80] and c.select(q, 2, 0, 0)[0].tolist() == [60, 80]
    assert 90 not in c.select(q, 199, 0, 0)[0].tolist()
    assert got[1:].tolist() == _ref_select(c, q, 4, 0, 0)[1:]


def test_select_planned_for_more_workgroups_than_a_grid_has_places(torch_cuda):  # noqa: F811
    # the most compute units that a cache may name, and a table with room for 2.2 million pages
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    c = Cache(torch, 3, [16 * 300], heads=1, group=2, D=128).fill()
    q = c.normal((1, 1, 2, 128))
    table = torch.full((1, 2_200_000), -1, dtype=torch.int32, device="cuda")
    table[:, : c.table.shape[1]] = c.table
    pages = B.make_pages(c.k_pool, c.v_pool, table, 2, compute_units=65536)
    ws = torch.empty((B.sablock_select_pages_workspace_bytes(pages),), dtype=torch.uint8, device="cuda")
    lst = torch.empty((1, 20), dtype=torch.int32, device="cuda")
    B.sablock_select_pages(pages, q, c.bounds, table, c.lengths, 20, lst, ws)
    assert lst.tolist() == _ref_select(c, q, 20, 1, 1)


@pytest.mark.parametrize("rows", [65536 * 16 + 1, 20000 * 16, 5000 * 16 + 7, 12001 * 16])
def test_select_among_many_pages(torch_cuda, rows):  # noqa: F811
    torch = torch_cuda
    c = Cache(torch, 3, [rows], heads=1, group=1, D=8)
    c.bounds.copy_(c.normal(c.bounds.shape).sort(dim=3).values)
    q = c.normal((1, 1, 1, 8))
    assert c.select(q, 700, 3, 5).tolist() == _ref_select(c, q, 700, 3, 5)


# ---- together ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,group,page", [("bf16", 4, 16), ("f32", 3, 32)])
def test_compress_then_decode_in_pages(torch_cuda, dtype, group, page):  # noqa: F811
    # the path into pages, then steps of a decoding loop, eager and captured, against a cache of plain rows in 64 bits
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B
    from paper_2510_22556_amd import synth

    dt, n, nl, H, D, L, W, budget, steps = _dt(torch, dtype), 2, 2, 2, 64, 1500, 16, 180, 6
    q, k, v = (synth.normal_torch(50 + i, i, (n, nl, h, m, D), "cuda", dt) for i, h, m in ((1, H * group, W), (2, H, L), (3, H, L)))
    seg = B.make_segments(np.concatenate([np.arange(0, L - W, 28), [L - W]] * n), np.arange(n + 1) * (-(-(L - W) // 28) + 1), "cuda")
    shape = B.make_shape(q, k, v)
    buf = B.Buffers(shape, seg, budget, "cuda")
    cap = -(-(budget + W + steps) // page)
    cache = B.PagedCache(n, nl, H * group, H, D, page, n * cap + 1, cap, dt, "cuda")
    cache.page_table.copy_(torch.randperm(n * cap + 1, device="cuda")[: n * cap].view(n, cap))
    B.compress(shape, q, k, v, seg, [1, 2, 4, 8], budget, buf, cache=cache)
    assert cache.lengths.tolist() == [budget + W] * n
    dense = B.Buffers(shape, seg, budget, "cuda")
    B.compress(shape, q, k, v, seg, [1, 2, 4, 8], budget, dense)
    assert torch.equal(dense.idx, buf.idx)
    keep_k, keep_v = (x.view(n, nl, H, budget + W, D).double().cpu() for x in (dense.k_out, dense.v_out))

    freq = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float32, device="cuda")
    positions = torch.full((n,), L, dtype=torch.int32, device="cuda")
    new = torch.zeros((n, nl, H * (group + 2), 1, D), dtype=dt, device="cuda")
    nq, nk, nv = new[:, :, : H * group], new[:, :, H * group: H * (group + 1)], new[:, :, H * (group + 1):]
    tokens = B.make_new_tokens(nk, nv, nq)
    rot = torch.empty((n, nl, H * group, 1, D), dtype=dt, device="cuda")
    outs = [torch.empty((n, nl, H * group, D), dtype=torch.float32, device="cuda") for _ in range(2)]
    lst = torch.empty((n * nl * H, 5), dtype=torch.int32, device="cuda")

    def step():
        cache.lengths.add_(1)
        B.sablock_append_paged(cache.pages, tokens, nk, nv, positions, freq, cache.page_table, cache.lengths, cache.k_pool, cache.v_pool,
                               q=nq, q_out=rot, bounds=cache.bounds)
        B.sablock_decode_paged(cache.pages, rot, cache.k_pool, cache.v_pool, cache.page_table, cache.lengths, outs[0], cache.ws)
        B.sablock_select_pages(cache.pages, rot, cache.bounds, cache.page_table, cache.lengths, 5, lst, cache.select_ws)
        B.sablock_decode_paged(cache.pages, rot, cache.k_pool, cache.v_pool, cache.page_table, cache.lengths, outs[1], cache.ws, page_list=lst)
        positions.add_(1)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for i in range(steps):
        new.copy_(synth.normal_torch(80 + i, 1, new.shape, "cuda", dt))
        if i == 2:                                              # from the third step on: captured, replayed
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(graph, stream=side):
                step()
        if i < 2:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        (rq, _), (rk, _) = _ref_append(type("C", (), {"torch": torch, "n": n}), nq, nk, [1] * n, [L + i] * n, freq.tolist(), D, False)
        keep_k = torch.cat([keep_k, rk.to(dt).double()], dim=3)
        keep_v = torch.cat([keep_v, nv.double().cpu()], dim=3)
        rows = keep_k.shape[3]
        assert cache.lengths.tolist() == [rows] * n
        # queries and keys are rounded once more than the reference's (half a step each, on either side of a tie): logits differ by that
        # of sum |q k| / sqrt(D) <= 10 at most, shares by as much; fp32 by its own arithmetic
        tol = 2 * 10 * torch.finfo(dt).eps * 5 + 2.0 ** -16 * 5
        for s in range(n):
            for l in range(nl):
                for h in range(H):
                    qs = rq[s, l, h * group: (h + 1) * group, 0].to(dt).double()
                    kk, vv = keep_k[s, l, h], keep_v[s, l, h]
                    got = outs[0][s, l, h * group: (h + 1) * group].double().cpu()
                    assert bool(((got - _attention(torch, qs, kk, vv)).abs() <= tol).all())
                    pages = lst[(s * nl + l) * H + h].tolist()
                    assert pages == sorted(pages) and pages[0] == 0 and pages[-1] == -(-rows // page) - 1 and len(set(pages)) == 5
                    at = torch.tensor([r for e in pages for r in range(e * page, min(rows, (e + 1) * page))])
                    got = outs[1][s, l, h * group: (h + 1) * group].double().cpu()
                    assert bool(((got - _attention(torch, qs, kk[at], vv[at])).abs() <= tol).all())


def test_calls_on_another_stream_and_twice_the_same(torch_cuda):  # noqa: F811
    # nothing is summed in an order that depends on who comes first: equal bits, on any stream, with any workspace contents
    torch = torch_cuda
    c = Cache(torch, 12, [3000, 100, 1], layers=1, heads=4, group=4, D=128).fill()
    q = c.normal((3, 1, 16, 128))
    want, lst = c.decode(q), c.select(q, 20)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for fill in (0, 0xFF, 0x7F):
        with torch.cuda.stream(side):
            again, lst2 = c.decode(q, ws_fill=fill), c.select(q, 20)
        side.synchronize()
        assert torch.equal(again, want) and torch.equal(lst, lst2)


def test_pools_beyond_two_to_the_31_elements(torch_cuda):  # noqa: F811
    # pages that lie more than 2^31 elements into the pool, in every call
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    D, page, n_pages = 128, 16, (2 ** 31 + 2 ** 26) // (128 * 16)
    k_pool, v_pool = (torch.zeros((1, n_pages, 1, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bounds = torch.zeros((1, n_pages, 1, 2, D), dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([40], dtype=torch.int32, device="cuda")
    pages = B.make_pages(k_pool, v_pool, table, 2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k, v = (torch.randn((1, 1, 1, 40, D), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    B.sablock_append_paged(pages, B.make_new_tokens(k, v, rotary_dim=0), k, v, None, None, table, lengths, k_pool, v_pool, bounds=bounds)
    assert torch.equal(k_pool[0, n_pages - 7, 0, :8], k[0, 0, 0, 32:]) and torch.equal(v_pool[0, n_pages - 1, 0], v[0, 0, 0, :16])
    assert torch.equal(bounds[0, n_pages - 1, 0, 1].float(), k[0, 0, 0, :16].float().amax(dim=0))
    q = torch.randn((1, 1, 2, D), generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.empty((1, 1, 2, D), dtype=torch.float32, device="cuda")
    ws = torch.empty((B.sablock_decode_paged_workspace_bytes(pages),), dtype=torch.uint8, device="cuda")
    B.sablock_decode_paged(pages, q, k_pool, v_pool, table, lengths, out, ws)
    ref = _attention(torch, q[0, 0].double().cpu(), k[0, 0, 0].double().cpu(), v[0, 0, 0].double().cpu())
    assert bool(((out[0, 0].double().cpu() - ref).abs() <= 2.0 ** -16 * 5).all())
    lst, sws = torch.empty((1, 2), dtype=torch.int32, device="cuda"), torch.empty((B.sablock_select_pages_workspace_bytes(pages),), dtype=torch.uint8, device="cuda")
    B.sablock_select_pages(pages, q, bounds, table, lengths, 2, lst, sws, n_first=0, n_last=1)
    up = [max(float(torch.maximum(x * bounds[0, int(i), 0, 0].double(), x * bounds[0, int(i), 0, 1].double()).sum()) for x in q[0, 0].double()) for i in table[0]]
    assert lst[0].tolist() == [0 if up[0] >= up[1] else 1, 2]

"""New tokens into the paged cache with a norm per head, against the formula in 64 bits: y = x w / sqrt(mean x^2 + eps), then rotated."""

import math

import pytest

from test_gpu_paged import NAN, Cache, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")


def _ref(torch, x, weight, per_head, eps, counts, positions, freq, R, interleaved):
    """Rows of x [n_seq, layers, heads, n_new, D] as they come out, in 64 bits, and |a| + |b| of every pair in front of the rotation."""
    x = x.double().cpu().clone()
    w = weight.double().cpu()
    w = w[None, :, :, None] if per_head else w[None, :, None, None]
    x = x * w / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)
    size = x.abs()
    for s in range(x.shape[0]):
        at = torch.arange(x.shape[3], dtype=torch.float64) + int(positions[s])
        for i in range(R // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
            t = at * float(freq[i])
            u, v = x[s, :, :, :, a].clone(), x[s, :, :, :, b].clone()
            x[s, :, :, :, a], x[s, :, :, :, b] = u * torch.cos(t) - v * torch.sin(t), v * torch.cos(t) + u * torch.sin(t)
            size[s, :, :, :, a] = size[s, :, :, :, b] = u.abs() + v.abs()
    return x, size


def _close(torch, got, ref, size):
    # In units of 2^-24 relative: the sum of squares, 8 in a lane and 6 lane steps, 14, half of that behind the root; the mean and eps 1, the root's
    # reciprocal 2; two products 2; cosine and sine 4; two products and their sum 3: 19 and a half, below 2^-19.  Then half a step of the type.
    half = torch.finfo(got.dtype).eps / 2
    err = (got.double().cpu() - ref).abs()
    assert bool((err <= half * ref.abs() * (1 + half) + 2.0 ** -19 * size).all()), float((err / (size + 1e-30)).max())


def _inputs(c, n_new, R):
    """q, k and v as views of one projection's output, heads of very different sizes, weights of both signs."""
    torch, n, H, G = c.torch, c.n, c.H, c.G
    qkv = (c.normal((n, n_new, c.L, H * (G + 2), c.D), torch.float32) * torch.exp(3 * c.normal((1, 1, 1, H * (G + 2), 1), torch.float32))).to(c.dt).permute(0, 2, 3, 1, 4)
    freq = torch.tensor([10000.0 ** (-2 * i / max(R, 1)) for i in range(R // 2)], dtype=torch.float32, device="cuda") if R else None
    return qkv[:, :, : H * G], qkv[:, :, H * G: H * (G + 1)], qkv[:, :, H * (G + 1):], freq


@pytest.mark.parametrize("D,R,interleaved,dtype,page,per_head", [
    (64, 64, False, "bf16", 16, False), (128, 128, False, "bf16", 64, True), (128, 64, True, "bf16", 32, False), (96, 96, True, "f32", 16, True), (96, 96, False, "bf16", 16, False),
    (256, 256, False, "f32", 256, False), (256, 256, False, "bf16", 128, True), (40, 16, False, "f32", 16, True), (72, 0, False, "bf16", 32, False), (8, 0, False, "f32", 16, True),
    (8, 0, False, "bf16", 16, False), (200, 96, False, "f32", 32, False)])
@pytest.mark.parametrize("n_new,lengths,counts", [(1, [1, 16, 17, 1000], None), (1, [5, 40, 0, 33], [1, 0, 1, -4]), (7, [7, 20, 64, 257], [7, 3, 7, 0]),
                                                  (130, [130, 400, 500, 131], None), (130, [1, 299, 300, 131], [130, 77, 300, 1])])
def test_append_normed(torch_cuda, D, R, interleaved, dtype, page, per_head, n_new, lengths, counts):  # noqa: F811
    torch = torch_cuda
    nl, H, G, eps = 2, 3, 2, 1e-5
    c = Cache(torch, D + R + n_new, lengths, layers=nl, heads=H, group=G, D=D, dtype=dtype, page=page, k_axes=(1, 3, 0, 2))
    B, n = c.B, c.n
    took = [min(n_new if counts is None else min(max(counts[s], 0), n_new), lengths[s]) for s in range(n)]
    after, c.lengths = c.lengths, c.lengths - torch.tensor(took, dtype=torch.int32, device="cuda")
    c.fill()
    c.lengths = after
    q, k, v, freq = _inputs(c, n_new, R)
    qw, kw = (c.normal((nl, heads, D) if per_head else (nl, D), torch.float32) for heads in (H * G, H))
    positions = torch.tensor([131071, 0, 7, 2 ** 30], dtype=torch.int32, device="cuda")
    q_out = torch.full((n, nl, H * G, n_new, D), 77.0, dtype=c.dt, device="cuda")
    tokens = B.make_new_tokens(k, v, q, rotary_dim=R, interleaved=interleaved)
    old = [t.clone() for t in (c.k_pool, c.v_pool, c.bounds)]
    B.sablock_append_normed_paged(c.pages, tokens, B.make_head_norms(eps, per_head), k, v, positions if R else None, freq, c.table, c.lengths, c.k_pool, c.v_pool,
                                  q=q, q_out=q_out, q_weight=qw, k_weight=kw, bounds=c.bounds,
                                  counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    f = [] if freq is None else freq.tolist()
    (rq, sq), (rk, sk) = (_ref(torch, x, w, per_head, eps, took, positions.tolist(), f, R, interleaved) for x, w in ((q, qw), (k, kw)))
    for s in range(n):
        _close(torch, q_out[s, :, :, : took[s]], rq[s, :, :, : took[s]], sq[s, :, :, : took[s]])
        assert bool((q_out[s, :, :, took[s]:] == 77.0).all())
        a, b = lengths[s] - took[s], lengths[s]
        if took[s]:
            _close(torch, c.rows(c.k_pool, s)[:, :, a:b].to(c.dt), rk[s, :, :, : took[s]], sk[s, :, :, : took[s]])
            assert torch.equal(c.rows(c.v_pool, s)[:, :, a:b], v[s, :, :, : took[s]].double().cpu())
        # the bounds are those of the rows that the pages now hold, untouched pages' and all other memory as before
        for i in range(a // page, -(-b // page) if took[s] else 0):
            at, m = int(c.table[s, i]), min(page, b - i * page)
            held = c.k_pool[:, at, :, :m].float()
            assert torch.equal(c.bounds[:, at, :, 0].float(), held.amin(dim=2)) and torch.equal(c.bounds[:, at, :, 1].float(), held.amax(dim=2))
            first = max(a - i * page, 0)
            for pool, was in ((c.k_pool, old[0]), (c.v_pool, old[1])):
                was[:, at, :, first:m] = pool[:, at, :, first:m]
            old[2][:, at] = c.bounds[:, at]
    bits = torch.int16 if c.dt == torch.bfloat16 else torch.int32
    for got, want in zip((c.k_pool, c.v_pool, c.bounds), old):
        assert torch.equal(got.contiguous().view(bits), want.contiguous().view(bits))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_new", [1, 37])
def test_heads_of_zeros_and_of_what_is_no_number(torch_cuda, dtype, n_new):  # noqa: F811
    # zeros stay zeros; squares beyond fp32 leave zeros; a tiny head is what eps makes of it; no number stays with its row and head
    torch = torch_cuda
    D, R, H = 64, 32, 4
    c = Cache(torch, 2, [n_new + 20], heads=H, group=1, D=D, dtype=dtype)
    q, k, v = (c.normal((1, 1, H, n_new, D)) for _ in range(3))
    freq = torch.tensor([100.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device="cuda")
    w = torch.ones((1, D), device="cuda")
    pos = torch.tensor([5], dtype=torch.int32, device="cuda")

    def call():
        out = torch.full(q.shape, 77.0, dtype=c.dt, device="cuda")
        c.B.sablock_append_normed_paged(c.pages, c.B.make_new_tokens(k, v, q, rotary_dim=R), c.B.make_head_norms(1e-6), k, v, pos, freq, c.table, c.lengths, c.k_pool,
                                        c.v_pool, q=q, q_out=out, q_weight=w, k_weight=w)
        return out

    clean = call()
    at = n_new // 2
    q[0, 0, 0, at] = 0.0
    q[0, 0, 1, at, 3] = 1e30
    q[0, 0, 2, at, 40] = NAN
    q[0, 0, 3, at] = 1e-10
    got = call()
    assert not got[0, 0, 0, at].any() and not got[0, 0, 1, at].any() and bool(torch.isnan(got[0, 0, 2, at]).all())
    # 1e-10 / sqrt(1e-20 + 1e-6): 1e-7 of a rotated pair of ones
    turned = got[0, 0, 3, at].double()
    assert bool((turned.abs() <= 1e-7 * 1.5).all()) and bool((turned[R:] / 1e-7 - 1).abs().max() <= 2.0 ** -7)
    got[0, 0, :, at] = clean[0, 0, :, at]
    assert torch.equal(got, clean)
    q[0, 0, 2, at, 40] = INF
    assert bool(torch.isnan(call()[0, 0, 2, at]).any())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_new", [1, 37])
def test_heads_as_large_as_the_type(torch_cuda, dtype, n_new, interleaved):  # noqa: F811
    # zeros whatever the weights are; an infinite element is no number, its head's others are zeros; the rows beside stay as they are, and V's do
    torch = torch_cuda
    D, R, H = 64, 32, 4
    c = Cache(torch, 3, [n_new + 20], heads=H, group=1, D=D, dtype=dtype)
    q, k, v = (c.normal((1, 1, H, n_new, D)) for _ in range(3))
    freq = torch.tensor([100.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device="cuda")
    w = torch.full((1, D), 8.0, device="cuda")
    pos = torch.tensor([5], dtype=torch.int32, device="cuda")

    def call():
        out = torch.full(q.shape, 77.0, dtype=c.dt, device="cuda")
        c.B.sablock_append_normed_paged(c.pages, c.B.make_new_tokens(k, v, q, rotary_dim=R, interleaved=interleaved), c.B.make_head_norms(1e-6), k, v, pos, freq,
                                        c.table, c.lengths, c.k_pool, c.v_pool, q=q, q_out=out, q_weight=w, k_weight=w)
        return out, c.rows(c.k_pool, 0)[0, :, 20:].clone(), c.rows(c.v_pool, 0)[0, :, 20:].clone()

    clean = call()
    at, most = n_new // 2, torch.finfo(c.dt).max
    q[0, 0, 0, at], q[0, 0, 2, at] = most, -most
    k[0, 0, 1, at], v[0, 0, 1, at], v[0, 0, 3, at, 7] = most, most, INF
    q[0, 0, 3, at, 60] = INF
    got = call()
    assert not got[0][0, 0, 0, at].any() and not got[0][0, 0, 2, at].any() and not got[1][1, at].any()
    assert bool(torch.isnan(got[0][0, 0, 3, at, 60])) and not got[0][0, 0, 3, at, :60].any()
    assert bool((got[2][1, at] == most).all()) and got[2][3, at, 7] == INF
    got[0][0, 0, [0, 2, 3], at], got[1][1, at], got[2][1, at], got[2][3, at, 7] = clean[0][0, 0, [0, 2, 3], at], clean[1][1, at], clean[2][1, at], clean[2][3, at, 7]
    for a, b in zip(got, clean):
        assert torch.equal(a, b)


def test_weights_of_ones_and_normed_rows_are_the_plain_append(torch_cuda):  # noqa: F811
    # rows whose mean square is one, eps too small to matter: the norm's factor is one to half a step of fp32, the append's result the other call's
    torch = torch_cuda
    n, H, D, n_new = 3, 2, 128, 9
    c = Cache(torch, 2, [40, 9, 100], heads=H, group=3, D=D, dtype="f32", page=32)
    q, k, v = (torch.sign(c.normal((n, 1, h, n_new, D))) for h in (3 * H, H, H))
    freq = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float32, device="cuda")
    pos, ones, tokens = torch.tensor([0, 70, 5000], dtype=torch.int32, device="cuda"), torch.ones((1, D), device="cuda"), c.B.make_new_tokens(k, v, q)
    a, b = torch.empty_like(q), torch.empty_like(q)
    c.B.sablock_append_paged(c.pages, tokens, k, v, pos, freq, c.table, c.lengths, c.k_pool, c.v_pool, q=q, q_out=a)
    want = c.k_pool.clone()
    c.B.sablock_append_normed_paged(c.pages, tokens, c.B.make_head_norms(1e-30), k, v, pos, freq, c.table, c.lengths, c.k_pool, c.v_pool, q=q, q_out=b, q_weight=ones,
                                    k_weight=ones)
    # the factor is off by one unit of 2^-23 at most; three more roundings of 2^-24 on either side; pairs of at most sqrt(2)
    tol = math.sqrt(2.0) * (2.0 ** -23 + 6 * 2.0 ** -24)
    assert bool(((a - b).abs() <= tol).all())
    for s in range(n):
        rows = int(c.lengths[s])
        was, c.k_pool = c.k_pool, want
        ref = c.rows(c.k_pool, s)[:, :, rows - n_new:]
        c.k_pool = was
        assert bool(((c.rows(c.k_pool, s)[:, :, rows - n_new:] - ref).abs() <= tol).all())


def test_normed_tokens_behind_a_full_table_and_without_queries(torch_cuda):  # noqa: F811
    # rows that the table has no room for are dropped, the last row in front of them stays
    torch = torch_cuda
    D, page = 64, 16
    c = Cache(torch, 3, [48, 48], heads=2, group=2, D=D, page=page)
    c.table = c.table[:, :3].contiguous()
    c.pages = c.B.make_pages(c.k_pool, c.v_pool, c.table, 4)
    c.fill()
    k, v = (c.normal((2, 1, 2, 5, D)) for _ in range(2))
    w = torch.ones((1, D), device="cuda")
    before = c.k_pool.clone()
    c.lengths = torch.tensor([50, 53], dtype=torch.int32, device="cuda")
    c.B.sablock_append_normed_paged(c.pages, c.B.make_new_tokens(k, v, rotary_dim=0), c.B.make_head_norms(1e-6), k, v, None, None, c.table, c.lengths, c.k_pool, c.v_pool,
                                    k_weight=w)
    ref, size = _ref(torch, k, w, False, 1e-6, [5, 5], [0, 0], [], 0, False)
    last = int(c.table[0, 2])
    _close(torch, c.k_pool[0, last, :, 13:], ref[0, 0, :, :3], size[0, 0, :, :3])
    before[0, last, :, 13:] = c.k_pool[0, last, :, 13:]
    assert torch.equal(c.k_pool.view(torch.int16), before.view(torch.int16))

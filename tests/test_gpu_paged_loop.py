"""A serving loop over the paged cache: a common prompt, prompts behind it, steps with normed and rotated tokens and attention that reads the common pages once; then
caches of their own, steps that gather weights, and evictions in between; eager, captured and replayed, against plain rows in 64 bits."""

import math

import pytest

from test_gpu_paged import Cache, _dt, torch_cuda  # noqa: F401
from test_gpu_paged_norm import _ref

pytestmark = pytest.mark.gpu


class Rows:
    """What the pages should hold: [layers, heads, rows, D] of K and V in 64 bits, and the rows' weights."""

    def __init__(self, torch, nl, H, D):
        self.torch = torch
        self.k, self.v = (torch.zeros((nl, H, 0, D), dtype=torch.float64) for _ in range(2))
        self.w = torch.zeros((nl, H, 0), dtype=torch.float64)

    def add(self, k, v):
        self.k, self.v = self.torch.cat([self.k, k], dim=2), self.torch.cat([self.v, v], dim=2)
        self.w = self.torch.cat([self.w, self.torch.zeros(k.shape[:3], dtype=self.torch.float64)], dim=2)

    def attend(self, q):
        """q [layers, heads, G, D]: outputs and shares summed over G."""
        share = self.torch.softmax(q @ self.k.transpose(-1, -2) / math.sqrt(q.shape[-1]), dim=-1)
        return share @ self.v, share.sum(dim=2)

    def keep(self, rows):
        """rows [layers][heads]: lists."""
        at = self.torch.tensor(rows, dtype=self.torch.long)
        take = lambda x: self.torch.gather(x, 2, at[..., None].expand(-1, -1, -1, x.shape[3]))  # noqa: E731
        self.k, self.v, self.w = take(self.k), take(self.v), self.torch.gather(self.w, 2, at)


@pytest.mark.parametrize("dtype,G,D,page", [("bf16", 4, 64, 16), ("f32", 3, 32, 32), ("bf16", 16, 128, 16)])
def test_serving_loop(torch_cuda, dtype, G, D, page):  # noqa: F811
    torch = torch_cuda
    from paper_2510_22556_amd import binding as B

    n, nl, H, dt, R, eps = 5, 2, 2, _dt(torch, dtype), D // 2, 1e-6
    common, most, keep, first, last = 3 * page, 4 * page, 2 * page + 5, 2, 6
    cap = 3 + 4 + 2
    cache = B.PagedCache(n, nl, H * G, H, D, page, 3 + n * 4 * cap, cap, dt, "cuda", weights=True, n_prefixes=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D)
    normal = lambda shape: torch.randn(shape, generator=gen, device="cuda").to(dt)  # noqa: E731
    free = torch.randperm(cache.k_pool.shape[1], generator=gen, device="cuda").to(torch.int32).tolist()
    shared, free = free[:3], free[3:]
    cache.page_table[:, :3] = torch.tensor(shared, dtype=torch.int32)
    for s in range(n):
        cache.page_table[s, 3:] = torch.tensor([free.pop() for _ in range(cap - 3)], dtype=torch.int32)
    freq = torch.tensor([10000.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device="cuda")
    qw, kw = (1 + 0.3 * torch.randn((nl, heads, D), generator=gen, device="cuda") for heads in (H * G, H))
    norms, held = B.make_head_norms(eps, per_head=True), [Rows(torch, nl, H, D) for _ in range(n)]

    def append(pages, table, lengths, m, positions, counts=None, q_out=None, new=None):
        """Tokens, and their rows as the cache should have them: normed and rotated in 64 bits, rounded once."""
        new = normal((table.shape[0], nl, H * (G + 2), m, D)) if new is None else new
        q, k, v = new[:, :, : H * G], new[:, :, H * G: H * (G + 1)], new[:, :, H * (G + 1):]
        tokens = B.make_new_tokens(k, v, None if q_out is None else q, rotary_dim=R)
        B.sablock_append_normed_paged(pages, tokens, norms, k, v, positions, freq, table, lengths, cache.k_pool, cache.v_pool, q=None if q_out is None else q, q_out=q_out,
                                      q_weight=qw, k_weight=kw, counts=counts, bounds=cache.bounds)
        return q, k, v

    def rows_of(x, weight, positions):
        m = x.shape[3]
        y, _ = _ref(torch, x, weight, True, eps, [m] * x.shape[0], positions, freq.tolist(), R, False)
        return y.to(dt).double()

    # the common prompt into three pages, once; then every sequence's own behind it, of several lengths
    one = B.make_pages(cache.k_pool, cache.v_pool, cache.page_table[:1].contiguous(), H * G)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    _, k, v = append(one, cache.page_table[:1].contiguous(), zero + common, common, zero)
    for s in range(n):
        held[s].add(rows_of(k, kw, [0])[0], v[0].double().cpu())
    counts = [most, 1, 0, 17, page]
    cache.lengths.copy_(torch.tensor([common + c for c in counts], dtype=torch.int32))
    _, k, v = append(cache.pages, cache.page_table, cache.lengths, most, torch.full((n,), common, dtype=torch.int32, device="cuda"), torch.tensor(counts, dtype=torch.int32, device="cuda"))
    ref = rows_of(k, kw, [common] * n)
    for s in range(n):
        held[s].add(ref[s, :, :, : counts[s]], v[s, :, :, : counts[s]].double().cpu())

    positions = cache.lengths.clone()
    new = torch.zeros((n, nl, H * (G + 2), 1, D), dtype=dt, device="cuda")
    q_out = torch.zeros((n, nl, H * G, 1, D), dtype=dt, device="cuda")
    out = torch.empty((n, nl, H * G, D), device="cuda")
    begin, n_pages = torch.tensor([0, 4, 5], dtype=torch.int32, device="cuda"), torch.tensor([3, 3], dtype=torch.int32, device="cuda")      # the last one by itself
    # Queries and keys are rounded once, as the reference's, but on either side of a tie: half a step on both sides of sum |q k| / sqrt(D) <= 12 at most; shares
    # by as much, and fp32 by its own arithmetic
    tol = 2 * 12 * torch.finfo(dt).eps + 2.0 ** -16

    def check(weighed):
        fp = positions.tolist()
        rk, rq = rows_of(new[:, :, H * G: H * (G + 1)], kw, [p - 1 for p in fp]), rows_of(new[:, :, : H * G], qw, [p - 1 for p in fp])
        for s in range(n):
            held[s].add(rk[s], new[s, :, :, 0][:, H * (G + 1):].double().cpu()[:, :, None])
            want, share = held[s].attend(rq[s, :, :, 0].view(nl, H, G, D))
            got = out[s].double().cpu().view(nl, H, G, D)
            assert bool(((got - want).abs() <= 5 * tol).all()), float((got - want).abs().max())
            assert int(cache.lengths[s]) == held[s].k.shape[2]
            if weighed:
                held[s].w += share
                r = torch.arange(held[s].k.shape[2])
                ids = table[s].cpu().long()[r // page]
                w = torch.stack([cache.weights[l].cpu()[ids, :, r % page].t() for l in range(nl)]).double()
                assert bool(((w - held[s].w).abs() <= held[s].w * tol + 2.0 ** -20).all()), float((w - held[s].w).abs().max())

    def token():
        new.copy_(normal(new.shape))

    # common pages read once
    for i in range(2):
        token()
        cache.lengths.add_(1)
        append(cache.pages, cache.page_table, cache.lengths, 1, positions, q_out=q_out, new=new)
        positions.add_(1)
        B.sablock_decode_prefix_paged(cache.pages, q_out, cache.k_pool, cache.v_pool, cache.page_table, cache.lengths, begin, n_pages, out, cache.prefix_ws)
        table = cache.page_table
        check(False)

    # pages of their own, whole sequences first, then the rows of most weight; steps in between
    table, spare = torch.full_like(cache.page_table, -1), cache.page_table.clone()
    lengths, rows_out = torch.zeros_like(cache.lengths), None

    def move(n_keep):
        nonlocal table, spare, rows_out
        for s in range(n):
            spare[s] = torch.tensor([free.pop() for _ in range(cap)], dtype=torch.int32)
        rows_out = torch.empty((n * nl * H, n_keep), dtype=torch.int32, device="cuda")
        B.sablock_evict_paged(cache.pages, table, cache.lengths, cache.weights, cache.k_pool, cache.v_pool, n_keep, spare, lengths, rows_out, cache.evict_ws,
                              n_first=first, n_last=last, bounds=cache.bounds)
        for s in range(n):
            rows, kept = held[s].k.shape[2], rows_out.view(n, nl, H, n_keep)[s].tolist()
            m = min(rows, n_keep)
            assert int(lengths[s]) == m
            weights = held[s].w
            for l in range(nl):
                for h in range(H):
                    x = kept[l][h]
                    assert x[:m] == sorted(set(x[:m])) and x[m:] == [-1] * (n_keep - m)
                    if rows > n_keep:
                        assert x[:first] == list(range(first)) and x[m - last: m] == list(range(rows - last, rows))
                        gone = sorted(set(range(rows)) - set(x[:m]))
                        least = min((float(weights[l, h, r]) for r in x[first: m - last]), default=math.inf)
                        assert max(float(weights[l, h, r]) for r in gone) <= least * (1 + 2 * tol) + 2.0 ** -19
            held[s].keep([[y[:m] for y in x] for x in kept])
        table, spare = spare.clone(), table
        cache.lengths.copy_(lengths)

    table = cache.page_table.clone()
    move(cap * page)
    cache.weights[:, shared] = 77.0                             # nobody's any more

    state = dict(table=table.clone())

    def step():
        cache.lengths.add_(1)
        append(cache.pages, state["table"], cache.lengths, 1, positions, q_out=q_out, new=new)
        positions.add_(1)
        B.sablock_decode_weighed_paged(cache.pages, q_out, cache.k_pool, cache.v_pool, state["table"], cache.lengths, cache.weights, out, cache.weighed_ws)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for i in range(8):
        token()
        state["table"].copy_(table)
        if i == 1:                                              # from the second step on: captured, replayed, over tables and lengths that change
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(graph, stream=side):
                step()
        if i == 0:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        check(True)
        if i in (2, 5):
            move(keep)

"""The paged cache's operators as a serving program calls them, and their plain forms.

A case is a dict of plain values.  ``op`` names the call:

  compact   the last step of the compression path, into pages instead of a dense cache
  append    new tokens into the pages: the position rotation of queries and keys on the way, page bounds kept up to date
  decode    attention of one new token per sequence over its pages
  sparse    the same over the pages that a score from the page bounds picks for every KV head: selection, then attention

A sequence's pages lie anywhere in the pool (a server's free list after some time); entries of the table behind its last
page are -1.  Keys have an offset per channel, as real keys do, which makes page bounds tell pages apart.  Lengths of a
batch are spread over (0, rows] by multiples of the golden ratio, the first sequence having the most rows.
"""

import math

import torch

own = False

DEV = "cuda:0"


def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "n_seq": 1, "layers": 1, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16}
    c.update(kw)
    return c


def listed():
    return [
        # one layer of an 8B model behind a short prompt, as a prefill that compresses layer by layer calls it
        _case("compact_layer_8k", "compact", length=8192, window=32, budget=992),
        # all layers behind a longer prompt in one call
        _case("compact_model_32k", "compact", layers=32, length=32768, window=32, budget=992),
        # three fp32 prompts of odd length, a large budget, large pages
        _case("compact_f32_odd", "compact", dtype="f32", n_seq=3, layers=2, q_heads=8, kv_heads=4, dim=64, page=64, length=5001,
              window=16, budget=2077),
        # the token that a single user's request makes, behind a compressed prompt of 131 072 tokens: latency alone
        _case("append_token", "append", n_new=1, ragged=False, rows=1300, position=131071, rotary=128, interleaved=False),
        # one token for each of a full batch
        _case("append_batch", "append", n_seq=256, n_new=1, ragged=False, rows=2000, position=60000, rotary=128, interleaved=False),
        # the next turn's prompts, padded to the longest; half of each head rotated, neighbouring pairs
        _case("append_prompts", "append", n_seq=5, n_new=4001, ragged=True, rows=6500, position=20000, rotary=64, interleaved=True,
              page=64),
        # one token over a compressed cache: what every later token costs
        _case("decode_compacted", "decode", rows=1056, ragged=False),
        # a batch of requests of all lengths
        _case("decode_batch", "decode", n_seq=64, rows=8192, ragged=True, page=64),
        # long contexts that were not compressed: the largest call
        _case("decode_4x128k", "decode", n_seq=4, rows=131072, ragged=False),
        # a small fp32 model with an odd group of heads, lengths of no round number
        _case("decode_f32_odd", "decode", dtype="f32", n_seq=6, q_heads=28, kv_heads=4, dim=64, rows=5003, ragged=True, page=32),
        # one token over the 128 of 8 192 pages that matter
        _case("sparse_128k", "sparse", rows=131072, ragged=False, pick=128, first=1, last=2),
        # a batch with a group of seven heads and larger pages
        _case("sparse_batch", "sparse", n_seq=16, q_heads=28, kv_heads=4, rows=32011, ragged=True, page=32, pick=64, first=1, last=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_ROWS = {"compact": 2 ** 18, "append": 2 ** 18, "decode": 2 ** 22, "sparse": 2 ** 22}      # rows x KV heads x sequences x layers


def draw(rng):
    op = rng.choice(["compact", "append", "decode", "decode", "sparse"])
    c = {"op": op, "dtype": "f32" if rng.random() < 0.2 else "bf16", "page": rng.choice([16, 16, 32, 64, 128])}
    c["kv_heads"] = rng.choice([1, 2, 4, 8, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 4, 5, 7, 8, 16] if op in ("decode", "append") else [1, 2, 4, 4, 5, 7, 8])
    c["dim"] = rng.choice([64, 96, 128, 128, 128, 256])
    c["layers"] = _log_int(rng, 1, 32) if op == "compact" else rng.choice([1, 1, 1, 2])
    c["n_seq"] = rng.choice([1, 1, 2, 3, 5, 8]) if op == "compact" else _log_int(rng, 1, 200)
    bytes_per = c["dim"] * (2 if c["dtype"] == "f32" else 1) / 128       # of a row, against one of the largest listed case
    problems = c["n_seq"] * c["layers"] * c["kv_heads"]
    per_key = max(1, c["q_heads"] / c["kv_heads"] / 4)                   # products of a row, likewise
    room = max(64, int(0.99 * MAX_ROWS[op] / bytes_per / problems / (per_key if op in ("decode", "sparse") else 1)))      # rows of a problem
    if op == "compact":
        c["window"] = rng.choice([8, 16, 32, 64])
        c["budget"] = max(1, min(_log_int(rng, 32, 4096), room - c["window"]))
        room_keys = max(c["budget"] + c["window"] + 1, int(2 ** 23 / bytes_per / problems))
        c["length"] = max(c["window"] + 1 + c["budget"] // 2, min(_log_int(rng, 256, 65536), room_keys))
        return c
    c["rows"] = max(1, min(_log_int(rng, 1, 131072), room))
    c["ragged"] = rng.random() < 0.6
    if op == "append":
        c["n_new"] = min(c["rows"], rng.choice([1, 1, 1, _log_int(rng, 2, 4000)]))
        c["position"] = c["rows"] + _log_int(rng, 1, 131072)
        c["rotary"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 0])
        c["interleaved"] = rng.random() < 0.3
    if op == "sparse":
        c["pick"] = _log_int(rng, 3, 300)
        c["first"], c["last"] = rng.choice([0, 1, 1]), rng.choice([1, 1, 2])
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _spread(most, n, ragged):
    """Numbers in [1, most], the first of them the largest."""
    return [max(1, math.ceil(most * (1 - s * 0.6180339887498949 % 1))) if ragged else most for s in range(n)]


def _lengths(case):
    if case["op"] == "compact":
        return [min(case["budget"], case["length"] - case["window"]) + case["window"]] * case["n_seq"]
    return _spread(case["rows"], case["n_seq"], case["ragged"])


def _counts(case):
    return [min(a, b) for a, b in zip(_spread(case["n_new"], case["n_seq"], case["ragged"]), _lengths(case))]


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, dtype=dtype, device=DEV)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _valid(state):
    """[n_seq, max_pages * page]: the rows that hold an entry."""
    table, case = state["table"], state["case"]
    return torch.arange(table.shape[1] * case["page"], device=DEV)[None] < state["lengths"][:, None]


def _bounds_of(state, dtype):
    """Least and largest key element of every page of every sequence over the rows that hold an entry."""
    table, pool = state["table"], state["k_pool"]
    k = pool[:, table.clamp(min=0).long()].to(dtype)                     # layer, sequence, page, head, row, element
    held = _valid(state).view(table.shape + (-1,))[None, :, :, None, :, None]
    return torch.stack([k.masked_fill(~held, math.inf).amin(dim=4), k.masked_fill(~held, -math.inf).amax(dim=4)], dim=4)


def _write_bounds(state, bounds, table, pages):
    """Bounds of the pages (sequence, page) for which `pages` holds to where the pool's page has them."""
    seq, page = pages.nonzero(as_tuple=True)
    state["bounds"][:, table[seq, page].long()] = bounds[:, seq, page].to(state["bounds"].dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, nl, hq, hkv, D, page = (case[x] for x in ("n_seq", "layers", "q_heads", "kv_heads", "dim", "page"))
    dt = _dtype(case)
    lengths = _lengths(case)
    need = [-(-r // page) for r in lengths]
    width, n_pages = max(need), sum(need) + 3                            # three pages belong to nobody
    free = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = free[at: at + m]
        at += m
    st = {"case": case, "table": table, "lengths": _int32(lengths)}
    offset = _normal(gen, (nl, 1, hkv, 1, D), torch.float32).to(dt)
    st["k_pool"] = _normal(gen, (nl, n_pages, hkv, page, D), dt) + offset
    st["v_pool"] = _normal(gen, (nl, n_pages, hkv, page, D), dt)
    if case["op"] == "compact":
        L, W = case["length"], case["window"]
        st["k"], st["v"] = _normal(gen, (n, nl, hkv, L, D), dt) + offset.view(1, nl, hkv, 1, D), _normal(gen, (n, nl, hkv, L, D), dt)
        keep = min(case["budget"], L - W)
        idx = torch.full((n * nl * hkv, case["budget"]), -1, dtype=torch.int32, device=DEV)
        for p in range(idx.shape[0]):
            idx[p, :keep] = torch.randperm(L - W, generator=gen, device=DEV)[:keep].sort().values.to(torch.int32)
        st["idx"] = idx
    if case["op"] in ("compact", "append", "sparse"):
        st["bounds"] = torch.zeros((nl, n_pages, hkv, 2, D), dtype=dt, device=DEV)
    if case["op"] == "append":
        counts = _counts(case)
        # q, k and v of the new tokens as a fused projection leaves them: token by token, all heads
        qkv = _normal(gen, (n, case["n_new"], nl, hq + 2 * hkv, D), dt).permute(0, 2, 3, 1, 4)
        st["q"], st["k"], st["v"] = qkv[:, :, :hq], qkv[:, :, hq: hq + hkv], qkv[:, :, hq + hkv:]
        st["counts"] = _int32(counts)
        st["positions"] = _int32([case["position"] + 17 * s for s in range(n)])
        R = case["rotary"]
        st["inv_freq"] = torch.tensor([500000.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device=DEV) if R else None
        st["q_out"] = torch.zeros((n, nl, hq, case["n_new"], D), dtype=dt, device=DEV)
        before = dict(st, lengths=st["lengths"] - st["counts"])          # bounds as they were before the tokens came
        held = _valid(before).view(n, width, page).any(dim=2)
        _write_bounds(st, _bounds_of(before, torch.float32), table, held)
    if case["op"] in ("decode", "sparse"):
        st["q"] = _normal(gen, (n, nl, hq, D), dt)
        st["out"] = torch.empty((n, nl, hq, D), dtype=torch.float32, device=DEV)
    if case["op"] == "sparse":
        _write_bounds(st, _bounds_of(st, torch.float32), table, table >= 0)
        st["list"] = torch.empty((n * nl * hkv, case["pick"]), dtype=torch.int32, device=DEV)
    if own:
        from paper_2510_22556_amd import binding as B

        st["pages"] = B.make_pages(st["k_pool"], st["v_pool"], table, hq)
        if case["op"] == "compact":
            W = case["window"]
            st["shape"] = B.make_shape(torch.empty((n, nl, hq, W, D), dtype=dt, device=DEV), st["k"], st["v"])
            st["len_out"] = torch.empty((n,), dtype=torch.int32, device=DEV)
        if case["op"] == "append":
            st["tokens"] = B.make_new_tokens(st["k"], st["v"], st["q"], rotary_dim=case["rotary"], interleaved=case["interleaved"])
        if case["op"] in ("decode", "sparse"):
            st["ws"] = torch.empty((B.sablock_decode_paged_workspace_bytes(st["pages"]),), dtype=torch.uint8, device=DEV)
        if case["op"] == "sparse":
            st["select_ws"] = torch.empty((B.sablock_select_pages_workspace_bytes(st["pages"]),), dtype=torch.uint8, device=DEV)
    return st


# ---- plain forms --------------------------------------------------------------------------------------------------------


def _rows_of(pool, table):
    """[n_seq, layers, heads, max_pages * page, D] in 32 bits: every sequence's rows in order."""
    x = pool[:, table.clamp(min=0).long()].float()
    return x.permute(1, 0, 3, 2, 4, 5).flatten(3, 4)


def _plain_compact(st):
    case = st["case"]
    n, nl, hkv, page = (case[x] for x in ("n_seq", "layers", "kv_heads", "page"))
    L, W = case["length"], case["window"]
    keep = min(case["budget"], L - W)
    recent = torch.arange(L - W, L, device=DEV).expand(n, nl, hkv, W)
    src = torch.cat([st["idx"][:, :keep].view(n, nl, hkv, keep).long(), recent], dim=3)[..., None].expand(-1, -1, -1, -1, case["dim"])
    r = torch.arange(keep + W, device=DEV)
    where = st["table"][:, r // page].long()                             # sequence, row
    for name, pool in (("k", "k_pool"), ("v", "v_pool")):
        rows = torch.gather(st[name], 3, src)                            # sequence, layer, head, row, element
        # advanced indices apart from each other: their axes (sequence, row) come first
        st[pool][:, where, :, (r % page).expand(n, -1)] = rows.permute(0, 3, 1, 2, 4)
    _write_bounds(st, _bounds_of(st, torch.float32), st["table"], st["table"] >= 0)
    return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"], "lengths": torch.full((n,), keep + W, dtype=torch.int32, device=DEV)}


def _rotated(x, cos, sin, R, interleaved):
    """x [.., tokens, D] with its first R elements rotated, in 32 bits."""
    x = x.float()
    if R == 0:
        return x
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2: R])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    head = torch.stack([ra, rb], dim=-1).flatten(-2) if interleaved else torch.cat([ra, rb], dim=-1)
    return torch.cat([head, x[..., R:]], dim=-1)


def _plain_append(st):
    case = st["case"]
    R, m, page, n = case["rotary"], case["n_new"], case["page"], case["n_seq"]
    cos = sin = None
    if R:
        angle = (st["positions"][:, None] + torch.arange(m, device=DEV)).double()[..., None] * st["inv_freq"].double()
        cos, sin = (f(angle).float()[:, None, None] for f in (torch.cos, torch.sin))       # sequence, -, -, token, pair
    live = torch.arange(m, device=DEV)[None] < st["counts"][:, None]
    q = _rotated(st["q"], cos, sin, R, case["interleaved"]).to(st["q_out"].dtype)
    st["q_out"].copy_(torch.where(live[:, None, None, :, None], q, st["q_out"]))
    k = _rotated(st["k"], cos, sin, R, case["interleaved"]).to(st["k_pool"].dtype)
    seq, j = live.nonzero(as_tuple=True)
    row = (st["lengths"] - st["counts"])[seq].long() + j
    where = st["table"][seq, row // page].long()
    st["k_pool"][:, where, :, row % page] = k[seq, :, :, j]
    st["v_pool"][:, where, :, row % page] = st["v"][seq, :, :, j]
    touched = torch.zeros(st["table"].shape, dtype=torch.bool, device=DEV)
    touched[seq, row // page] = True
    _write_bounds(st, _bounds_of(st, torch.float32), st["table"], touched)
    return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"]}


def _plain_select(st):
    """Listed pages [problems, pick], ascending, -1 behind the last."""
    case, table = st["case"], st["table"]
    n, nl, hkv, D, pick = (case[x] for x in ("n_seq", "layers", "kv_heads", "dim", "pick"))
    b = st["bounds"][:, table.clamp(min=0).long()].double().permute(1, 0, 3, 4, 2, 5)      # sequence, layer, head, bound, page, element
    q = st["q"].view(n, nl, hkv, -1, D).double()
    # in 64 bits: the order of two pages is a whole number, and their scores may lie close
    score = torch.matmul(q.clamp(min=0), b[:, :, :, 1].transpose(-1, -2).contiguous()) + torch.matmul(q.clamp(max=0), b[:, :, :, 0].transpose(-1, -2).contiguous())
    score = score.amax(dim=3).float()                                    # sequence, layer, head, page
    pages = ((st["lengths"] + case["page"] - 1) // case["page"])[:, None, None, None]
    i = torch.arange(table.shape[1], device=DEV)
    score = score.masked_fill((i < case["first"]) | (i >= pages - case["last"]), math.inf).masked_fill(i >= pages, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :pick]
    if best.shape[-1] < pick:
        best = torch.cat([best, best.new_full(best.shape[:-1] + (pick - best.shape[-1],), table.shape[1])], dim=-1)
    best = best.masked_fill(best >= pages, table.shape[1]).sort(dim=-1).values
    return best.masked_fill(best >= table.shape[1], -1).to(torch.int32).view(n * nl * hkv, pick)


def _plain_attention(st, k, v, held):
    """k, v [n_seq, layers, heads, rows, D] in 32 bits, held [n_seq, layers, heads, rows]: one query per head over the held rows."""
    case = st["case"]
    n, nl, hkv, D = (case[x] for x in ("n_seq", "layers", "kv_heads", "dim"))
    q = st["q"].view(n, nl, hkv, -1, D).float()
    x = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D)
    x = x.masked_fill(~held[:, :, :, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    den = e.sum(dim=-1, keepdim=True)
    out = torch.matmul(e, v) / torch.where(den > 0, den, 1.0)
    return out.view(n, nl, -1, D)


def _plain_decode(st):
    held = _valid(st)[:, None, None].expand(-1, st["case"]["layers"], st["case"]["kv_heads"], -1)
    return {"out": _plain_attention(st, _rows_of(st["k_pool"], st["table"]), _rows_of(st["v_pool"], st["table"]), held)}


def _plain_sparse(st):
    case = st["case"]
    n, nl, hkv, page, pick = (case[x] for x in ("n_seq", "layers", "kv_heads", "page", "pick"))
    listed_pages = _plain_select(st)
    at = listed_pages.view(n, nl, hkv, pick).long()
    where = torch.gather(st["table"].long()[:, None, None].expand(-1, nl, hkv, -1), 3, at.clamp(min=0)).clamp(min=0)
    layer, head = torch.arange(nl, device=DEV)[None, :, None, None], torch.arange(hkv, device=DEV)[None, None, :, None]
    k, v = (st[p][layer, where, head].float().flatten(3, 4) for p in ("k_pool", "v_pool"))
    row = at[..., None] * page + torch.arange(page, device=DEV)
    held = ((at[..., None] >= 0) & (row < st["lengths"].view(n, 1, 1, 1, 1))).flatten(3, 4)
    return {"list": listed_pages, "out": _plain_attention(st, k, v, held)}


def run(state):
    st, case = state, state["case"]
    if not own:
        return {"compact": _plain_compact, "append": _plain_append, "decode": _plain_decode, "sparse": _plain_sparse}[case["op"]](st)
    from paper_2510_22556_amd import binding as B

    pages, table = st["pages"], st["table"]
    if case["op"] == "compact":
        B.sablock_compact_paged(st["shape"], st["k"], st["v"], st["idx"], case["budget"], True, pages, table, st["k_pool"], st["v_pool"],
                                bounds=st["bounds"], lengths_out=st["len_out"])
        return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"], "lengths": st["len_out"]}
    if case["op"] == "append":
        B.sablock_append_paged(pages, st["tokens"], st["k"], st["v"], st["positions"], st["inv_freq"], table, st["lengths"], st["k_pool"],
                               st["v_pool"], q=st["q"], q_out=st["q_out"], counts=st["counts"], bounds=st["bounds"])
        return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"]}
    if case["op"] == "decode":
        B.sablock_decode_paged(pages, st["q"], st["k_pool"], st["v_pool"], table, st["lengths"], st["out"], st["ws"])
        return {"out": st["out"]}
    B.sablock_select_pages(pages, st["q"], st["bounds"], table, st["lengths"], case["pick"], st["list"], st["select_ws"],
                           n_first=case["first"], n_last=case["last"])
    B.sablock_decode_paged(pages, st["q"], st["k_pool"], st["v_pool"], table, st["lengths"], st["out"], st["ws"], page_list=st["list"])
    return {"list": st["list"], "out": st["out"]}


# ---- the definitions in 64 bits, one sequence and one row or page at a time where that is affordable ---------------------


def _exact_attention(q, k, v):
    """q [layers, heads, G, D], k, v [layers, heads, rows, D]."""
    w = torch.softmax(torch.matmul(q, k.transpose(-1, -2).contiguous()) * q.shape[-1] ** -0.5, dim=-1)
    return torch.matmul(w, v).flatten(1, 2)


def exact(case, seed):
    st = prepare(case, seed)
    n, nl, hkv, D, page = (case[x] for x in ("n_seq", "layers", "kv_heads", "dim", "page"))
    lengths, table = _lengths(case), st["table"].tolist()
    if case["op"] in ("compact", "append"):
        if n * nl * (lengths[0] if case["op"] == "compact" else case["n_new"]) > 2 ** 17:
            return None
        kp, vp, bounds = st["k_pool"].double(), st["v_pool"].double(), st["bounds"].double()
        if case["op"] == "compact":
            kept = st["idx"].view(n, nl, hkv, -1)
            keep = min(case["budget"], case["length"] - case["window"])
        else:
            q_out = st["q_out"].double()
        for s in range(n):
            if case["op"] == "compact":
                first, count = 0, lengths[s]
                tail = torch.arange(case["length"] - case["window"], case["length"], device=DEV)
                new_k, new_v = (torch.stack([torch.stack([st[x][s, l, h].double()[torch.cat([kept[s, l, h, :keep].long(), tail])] for h in range(hkv)])
                                             for l in range(nl)]) for x in ("k", "v"))
            else:
                count = _counts(case)[s]
                first = lengths[s] - count
                new_k, new_q = (st[x][s, :, :, :count].double().clone() for x in ("k", "q"))
                new_v = st["v"][s, :, :, :count].double()
                R = case["rotary"]
                place = torch.arange(count, device=DEV, dtype=torch.float64) + float(st["positions"][s])
                for i in range(R // 2):
                    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
                    turn = torch.polar(torch.ones_like(place), place * float(st["inv_freq"][i]))
                    for x in (new_k, new_q):                             # a pair as a complex number, turned by the angle
                        z = torch.complex(x[..., a], x[..., b]) * turn
                        x[..., a], x[..., b] = z.real, z.imag
                q_out[s, :, :, :count] = new_q
            for r0 in range(first // page * page, first + count, page):
                page_id = table[s][r0 // page]
                lo, hi = max(first, r0), min(first + count, r0 + page)
                kp[:, page_id, :, lo - r0: hi - r0] = new_k[:, :, lo - first: hi - first]
                vp[:, page_id, :, lo - r0: hi - r0] = new_v[:, :, lo - first: hi - first]
                held = kp[:, page_id, :, : hi - r0]
                bounds[:, page_id, :, 0], bounds[:, page_id, :, 1] = held.amin(dim=2), held.amax(dim=2)
        out = {"k_pool": kp, "v_pool": vp, "bounds": bounds}
        if case["op"] == "compact":
            return dict(out, lengths=_int32(lengths))
        return {"q": q_out, **out}
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    chosen = []
    for s in range(n):
        ids = table[s][: -(-lengths[s] // page)]
        q = st["q"][s].double().view(nl, hkv, -1, D)
        if case["op"] == "decode":
            ids_t = torch.tensor(ids, device=DEV)
            k, v = (st[p][:, ids_t].double().transpose(1, 2).flatten(2, 3)[:, :, : lengths[s]] for p in ("k_pool", "v_pool"))
            out[s] = _exact_attention(q, k, v)
            continue
        b = st["bounds"][:, torch.tensor(ids, device=DEV)].double()      # layer, page, head, bound, element
        for l in range(nl):
            for h in range(hkv):
                most = torch.full((len(ids),), -math.inf, dtype=torch.float64, device=DEV)
                for g in range(q.shape[2]):
                    x = q[l, h, g]
                    most = torch.maximum(most, torch.maximum(x * b[l, :, h, 0], x * b[l, :, h, 1]).sum(dim=-1))
                values = most.float().tolist()
                forced = sorted(set(range(min(case["first"], len(ids)))) | set(range(max(0, len(ids) - case["last"]), len(ids))))
                if len(ids) <= case["pick"]:
                    pages = list(range(len(ids)))
                else:
                    rest = sorted((i for i in range(len(ids)) if i not in forced), key=lambda i: (-values[i], i))
                    pages = sorted(forced + rest[: case["pick"] - len(forced)])
                chosen.append(pages + [-1] * (case["pick"] - len(pages)))
                rows = [p * page + r for p in pages for r in range(page) if p * page + r < lengths[s]]
                where = torch.tensor([ids[r // page] for r in rows], device=DEV), torch.tensor([r % page for r in rows], device=DEV)
                k, v = (st[p][l, where[0], h, where[1]].double()[None, None] for p in ("k_pool", "v_pool"))
                G = q.shape[2]
                out[s, l, h * G: (h + 1) * G] = _exact_attention(q[l, h][None, None], k, v)[0]
    return {"out": out} if case["op"] == "decode" else {"list": _int32(chosen), "out": out}


# ---- what the calls cannot do without -----------------------------------------------------------------------------------


def work(case):
    elt = 4 if case["dtype"] == "f32" else 2
    n, nl, hq, hkv, D, page = (case[x] for x in ("n_seq", "layers", "q_heads", "kv_heads", "dim", "page"))
    lengths = _lengths(case)
    pages = [-(-r // page) for r in lengths]
    row = nl * hkv * D * elt                                             # bytes of K of one row of all problems of a sequence
    if case["op"] == "compact":
        keep = lengths[0] - case["window"]
        return {"bytes": sum(4 * row * r for r in lengths) + 2 * row * sum(pages) + 4 * n * nl * hkv * keep + 4 * sum(pages) + 4 * n,
                "flops": 2.0 * nl * hkv * D * sum(lengths)}
    if case["op"] == "append":
        counts = _counts(case)
        touched = sum(-(-r // page) - (r - c) // page for r, c in zip(lengths, counts))
        merged = sum((r - c) % page > 0 for r, c in zip(lengths, counts))                  # pages whose bounds are read as well
        tokens = sum(counts)
        return {"bytes": tokens * (4 * row + 2 * nl * hq * D * elt) + 2 * row * (touched + merged) + 4 * touched + 12 * n,
                "flops": tokens * nl * (hq + hkv) * 3.0 * case["rotary"] + 2.0 * tokens * nl * hkv * D}
    q = n * nl * hq * D * (elt + 4)
    if case["op"] == "decode":
        return {"bytes": 2 * row * sum(lengths) + q + 4 * sum(pages) + 4 * n, "flops": 4.0 * nl * hq * D * sum(lengths)}
    picked = sum(min(r, case["pick"] * page) for r in lengths)
    return {"bytes": 2 * row * (picked + sum(pages)) + q + n * nl * hq * D * elt + 4 * sum(pages) + 4 * n + 4 * n * nl * hkv * case["pick"],
            "flops": 4.0 * nl * hq * D * (picked + sum(pages))}

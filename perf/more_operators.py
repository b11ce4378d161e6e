"""More operators of the paged cache as a serving program calls them, and their plain forms.

A case is a dict of plain values.  ``op`` names the call:

  normed    new tokens into the pages: queries and keys divided by their root mean square, weighted and rotated on the way
  weighed   attention of one new token per sequence, and every row's share of it added to what the row has gathered so far
  evict     the rows that gathered the most, the first and the last ones into new pages, in their order
  prefix    attention of one new token per sequence where sequences have their first pages in common, read once for all

A sequence's pages lie anywhere in the pool (a server's free list after some time); entries of the table behind its last
page are -1.  Keys have an offset per channel, as real keys do.  Lengths of a batch are spread over (0, rows] by multiples of
the golden ratio, the first sequence having the most rows.
"""

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "n_seq": 1, "layers": 1, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "ragged": False}
    c.update(kw)
    return c


def listed():
    return [
        # the token that a single user's request makes, behind a compressed prompt of 131 072 tokens: latency alone
        _case("normed_token", "normed", n_new=1, rows=1300, position=131071, rotary=128, interleaved=False, per_head=False),
        # one token for each of a full batch, every head with a weight of its own
        _case("normed_batch", "normed", n_seq=256, n_new=1, rows=2000, position=60000, rotary=128, interleaved=False, per_head=True),
        # the next turn's prompts, padded to the longest
        _case("normed_prompts", "normed", n_seq=5, n_new=4001, ragged=True, rows=6500, position=20000, rotary=128, interleaved=False, per_head=False,
              page=64),
        # a small fp32 model with an odd group of heads; half of each head rotated, neighbouring pairs
        _case("normed_f32_odd", "normed", dtype="f32", n_seq=3, q_heads=28, kv_heads=4, dim=64, n_new=777, ragged=True, rows=5003, position=9000, rotary=32,
              interleaved=True, per_head=True, page=32),
        # one token over a compressed cache: what every later token costs
        _case("weighed_compacted", "weighed", rows=1056, fresh=1, decay=1.0),
        # a batch of requests of all lengths, what was gathered long ago counting less
        _case("weighed_batch", "weighed", n_seq=64, rows=8192, ragged=True, page=64, fresh=1, decay=0.99),
        # a small fp32 model with an odd group of heads, lengths of no round number, several rows that nobody has weighed yet
        _case("weighed_f32_odd", "weighed", dtype="f32", n_seq=6, q_heads=28, kv_heads=4, dim=64, rows=5003, ragged=True, page=32, fresh=40, decay=1.0),
        # one layer of an 8B model whose cache has grown by 128 rows beyond its budget
        _case("evict_layer", "evict", rows=1184, keep=1056, first=4, last=256),
        # all layers of four sequences of all lengths in one call
        _case("evict_model", "evict", n_seq=4, layers=32, rows=4352, ragged=True, keep=2048, first=4, last=512),
        # a few requests behind a short system prompt
        _case("prefix_8x2k", "prefix", n_seq=8, prefixes=1, prefix_rows=2048, rows=300, ragged=True),
        # a full batch of questions about one long document: the largest call
        _case("prefix_64x32k", "prefix", n_seq=64, prefixes=1, prefix_rows=32768, rows=2048, ragged=True, page=64),
        # a small fp32 model, three documents with several questions each
        _case("prefix_f32_groups", "prefix", dtype="f32", n_seq=13, q_heads=28, kv_heads=4, dim=64, prefixes=3, prefix_rows=5024, rows=333, ragged=True,
              page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_ROWS = {"normed": 2 ** 18, "weighed": 2 ** 22, "evict": 2 ** 21, "prefix": 2 ** 24}        # rows x KV heads x sequences x layers


def draw(rng):
    op = rng.choice(["normed", "weighed", "evict", "prefix", "prefix"])
    c = {"op": op, "dtype": "f32" if rng.random() < 0.2 else "bf16", "page": rng.choice([16, 16, 32, 64, 128])}
    c["kv_heads"] = rng.choice([1, 2, 4, 8, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    c["dim"] = rng.choice([64, 96, 128, 128, 128, 256])
    c["layers"] = _log_int(rng, 1, 32) if op == "evict" else rng.choice([1, 1, 1, 2])
    c["n_seq"] = rng.choice([1, 1, 2, 3, 5, 8]) if op == "evict" else _log_int(rng, 2 if op == "prefix" else 1, 200)
    bytes_per = c["dim"] * (2 if c["dtype"] == "f32" else 1) / 128       # of a row, against one of the largest listed case
    problems = c["n_seq"] * c["layers"] * c["kv_heads"]
    per_key = max(1, c["q_heads"] / c["kv_heads"] / 4)                   # query heads of a row, likewise
    if c["dtype"] == "f32" and op == "prefix":
        per_key *= 4                                                     # products of 32 bits
    room = max(64, int(0.99 * MAX_ROWS[op] / bytes_per / problems / (1 if op == "evict" else per_key)))      # rows of a problem
    c["rows"] = max(1, min(_log_int(rng, 1, 131072), room))
    c["ragged"] = rng.random() < 0.6
    if op == "normed":
        c["n_new"] = min(c["rows"], rng.choice([1, 1, 1, _log_int(rng, 2, 4000)]))
        c["position"] = c["rows"] + _log_int(rng, 1, 131072)
        c["rotary"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 0])
        c["interleaved"] = rng.random() < 0.3
        c["per_head"] = rng.random() < 0.4
    if op == "weighed":
        c["fresh"] = min(c["rows"], rng.choice([0, 1, 1, 1, _log_int(rng, 2, 600)]))
        c["decay"] = rng.choice([1.0, 1.0, 0.98, 0.5])
    if op == "evict":
        c["rows"] = max(c["rows"], 24)
        c["keep"] = max(8, min(_log_int(rng, 16, 8192), c["rows"] - c["rows"] // 16))
        c["first"], c["last"] = rng.choice([0, 4, 4]), rng.choice([1, c["keep"] // 8, c["keep"] // 2])
        c["first"] = min(c["first"], c["keep"] - c["last"])
    if op == "prefix":
        c["prefixes"] = min(c["n_seq"], rng.choice([1, 1, 1, 2, 5, _log_int(rng, 2, 40)]))
        c["rows"] = min(c["rows"], 8192, max(1, room // 2))
        c["prefix_rows"] = max(c["page"], min(_log_int(rng, 64, 131072), room - c["rows"]))
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _spread(most, n, ragged):
    """Numbers in [1, most], the first of them the largest."""
    return [max(1, math.ceil(most * (1 - s * 0.6180339887498949 % 1))) if ragged else most for s in range(n)]


def _groups(case):
    """Where the sequences of each prefix begin (and the last ones end), and each prefix's pages."""
    m = case["prefixes"]
    share, begin, at = _spread(3 * case["n_seq"], m, True), [0], 0       # uneven, none empty
    for i, x in enumerate(share, 1):
        at += x
        begin.append(min(max(begin[-1] + 1, case["n_seq"] * at // sum(share)), case["n_seq"] - (m - i)))
    pages = max(1, case["prefix_rows"] // case["page"])
    return begin, _spread(pages, m, case["ragged"])


def _prefix_pages(case):
    """Pages in front of each sequence's own rows."""
    if case["op"] != "prefix":
        return [0] * case["n_seq"]
    begin, pages = _groups(case)
    return [pages[i] for i in range(len(pages)) for _ in range(begin[i], begin[i + 1])]


def _lengths(case):
    return [n + m * case["page"] for n, m in zip(_spread(case["rows"], case["n_seq"], case["ragged"]), _prefix_pages(case))]


def _counts(case):
    return [min(a, b) for a, b in zip(_spread(case["n_new"], case["n_seq"], case["ragged"]), _lengths(case))]


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, dtype=dtype, device=DEV)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _valid(state, table="table", lengths="lengths"):
    """[n_seq, max_pages * page]: the rows that hold an entry."""
    return torch.arange(state[table].shape[1] * state["case"]["page"], device=DEV)[None] < state[lengths][:, None]


def _bounds_of(state, dtype, table="table", lengths="lengths"):
    """Least and largest key element of every page of every sequence over the rows that hold an entry."""
    t = state[table]
    k = state["k_pool"][:, t.clamp(min=0).long()].to(dtype)              # layer, sequence, page, head, row, element
    held = _valid(state, table, lengths).view(t.shape + (-1,))[None, :, :, None, :, None]
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
    lengths, common = _lengths(case), _prefix_pages(case)
    need = [-(-r // page) for r in lengths]
    kept = [-(-min(r, case["keep"]) // page) for r in lengths] if case["op"] == "evict" else [0] * n
    begin, of_prefix = _groups(case) if case["op"] == "prefix" else ([], [])
    width, n_pages = max(need), sum(need) - sum(common) + sum(of_prefix) + sum(kept) + 3       # three pages belong to nobody
    free = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table, after = (torch.full((n, width), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    at = 0
    for i, m in enumerate(of_prefix):
        table[begin[i]: begin[i + 1], :m] = free[at: at + m]
        at += m
    for s in range(n):
        m = need[s] - common[s]
        table[s, common[s]: need[s]] = free[at: at + m]
        after[s, : kept[s]] = free[at + m: at + m + kept[s]]
        at += m + kept[s]
    st = {"case": case, "table": table, "lengths": _int32(lengths)}
    offset = _normal(gen, (nl, 1, hkv, 1, D), torch.float32).to(dt)
    st["k_pool"] = _normal(gen, (nl, n_pages, hkv, page, D), dt) + offset
    st["v_pool"] = _normal(gen, (nl, n_pages, hkv, page, D), dt)
    if case["op"] in ("normed", "evict"):
        st["bounds"] = torch.zeros((nl, n_pages, hkv, 2, D), dtype=dt, device=DEV)
    if case["op"] in ("weighed", "evict"):
        # a few rows gather most of the weight, others next to none
        st["weights"] = torch.exp(2 * _normal(gen, (nl, n_pages, hkv, page), torch.float32) - 4)
    if case["op"] == "normed":
        # q, k and v of the new tokens as a fused projection leaves them: token by token, all heads; heads of different sizes
        size = torch.exp(_normal(gen, (1, 1, 1, hq + 2 * hkv, 1), torch.float32))
        qkv = (_normal(gen, (n, case["n_new"], nl, hq + 2 * hkv, D), torch.float32) * size).to(dt).permute(0, 2, 3, 1, 4)
        st["q"], st["k"], st["v"] = qkv[:, :, :hq], qkv[:, :, hq: hq + hkv], qkv[:, :, hq + hkv:]
        for name, heads in (("q_weight", hq), ("k_weight", hkv)):
            shape = (nl, heads, D) if case["per_head"] else (nl, D)
            st[name] = 1 + 0.2 * _normal(gen, shape, torch.float32)
        st["counts"] = _int32(_counts(case))
        st["positions"] = _int32([case["position"] + 17 * s for s in range(n)])
        R = case["rotary"]
        st["inv_freq"] = torch.tensor([500000.0 ** (-2 * i / R) for i in range(R // 2)], dtype=torch.float32, device=DEV) if R else None
        st["q_out"] = torch.zeros((n, nl, hq, case["n_new"], D), dtype=dt, device=DEV)
        st["before"] = st["lengths"] - st["counts"]                      # bounds as they were before the tokens came
        _write_bounds(st, _bounds_of(st, torch.float32, lengths="before"), table, _valid(st, lengths="before").view(n, width, page).any(dim=2))
    if case["op"] in ("weighed", "prefix"):
        st["q"] = _normal(gen, (n, nl, hq, D), dt)
        st["out"] = torch.empty((n, nl, hq, D), dtype=torch.float32, device=DEV)
    if case["op"] == "weighed":
        st["counts"] = _int32([min(case["fresh"], r) for r in lengths])
    if case["op"] == "evict":
        st["after"] = after
        st["len_out"] = torch.empty((n,), dtype=torch.int32, device=DEV)
        st["rows_out"] = torch.empty((n * nl * hkv, case["keep"]), dtype=torch.int32, device=DEV)
        _write_bounds(st, _bounds_of(st, torch.float32), table, table >= 0)
    if case["op"] == "prefix":
        st["begin"], st["prefix_pages"] = _int32(begin), _int32(of_prefix)
    if own:
        from paper_2510_22556_amd import binding as B

        st["pages"] = B.make_pages(st["k_pool"], st["v_pool"], table, hq)
        if case["op"] == "normed":
            st["tokens"] = B.make_new_tokens(st["k"], st["v"], st["q"], rotary_dim=case["rotary"], interleaved=case["interleaved"])
            st["norms"] = B.make_head_norms(EPS, per_head=case["per_head"])
        else:
            size = {"weighed": lambda: B.sablock_decode_weighed_paged_workspace_bytes(st["pages"]),
                    "evict": lambda: B.sablock_evict_paged_workspace_bytes(st["pages"]),
                    "prefix": lambda: B.sablock_decode_prefix_paged_workspace_bytes(st["pages"], len(of_prefix))}[case["op"]]()
            st["ws"] = torch.empty((size,), dtype=torch.uint8, device=DEV)
    return st


# ---- plain forms --------------------------------------------------------------------------------------------------------


def _rows_of(pool, table):
    """[n_seq, layers, heads, max_pages * page, D] in 32 bits: every sequence's rows in order."""
    x = pool[:, table.clamp(min=0).long()].float()
    return x.permute(1, 0, 3, 2, 4, 5).flatten(3, 4)


def _normed(x, weight, per_head):
    """x [n_seq, layers, heads, tokens, D] over its root mean square, weighted, in 32 bits."""
    x = x.float()
    w = weight[None, :, :, None] if per_head else weight[None, :, None, None]
    return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w


def _rotated(x, cos, sin, R, interleaved):
    """x [.., tokens, D] with its first R elements rotated, in 32 bits."""
    if R == 0:
        return x
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2: R])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    head = torch.stack([ra, rb], dim=-1).flatten(-2) if interleaved else torch.cat([ra, rb], dim=-1)
    return torch.cat([head, x[..., R:]], dim=-1)


def _plain_normed(st):
    case = st["case"]
    R, m, page = case["rotary"], case["n_new"], case["page"]
    cos = sin = None
    if R:
        angle = (st["positions"][:, None] + torch.arange(m, device=DEV)).double()[..., None] * st["inv_freq"].double()
        cos, sin = (f(angle).float()[:, None, None] for f in (torch.cos, torch.sin))       # sequence, -, -, token, pair
    live = torch.arange(m, device=DEV)[None] < st["counts"][:, None]
    q = _rotated(_normed(st["q"], st["q_weight"], case["per_head"]), cos, sin, R, case["interleaved"]).to(st["q_out"].dtype)
    st["q_out"].copy_(torch.where(live[:, None, None, :, None], q, st["q_out"]))
    k = _rotated(_normed(st["k"], st["k_weight"], case["per_head"]), cos, sin, R, case["interleaved"]).to(st["k_pool"].dtype)
    seq, j = live.nonzero(as_tuple=True)
    row = (st["lengths"] - st["counts"])[seq].long() + j
    where = st["table"][seq, row // page].long()
    st["k_pool"][:, where, :, row % page] = k[seq, :, :, j]
    st["v_pool"][:, where, :, row % page] = st["v"][seq, :, :, j]
    touched = torch.zeros(st["table"].shape, dtype=torch.bool, device=DEV)
    touched[seq, row // page] = True
    _write_bounds(st, _bounds_of(st, torch.float32), st["table"], touched)
    return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"]}


def _plain_shares(st):
    """Softmax of one query per head over a sequence's rows [n_seq, layers, KV heads, G, rows] in 32 bits."""
    case = st["case"]
    n, nl, hkv, D = (case[x] for x in ("n_seq", "layers", "kv_heads", "dim"))
    q = st["q"].view(n, nl, hkv, -1, D).float()
    x = torch.matmul(q, _rows_of(st["k_pool"], st["table"]).transpose(-1, -2)) / math.sqrt(D)
    x = x.masked_fill(~_valid(st)[:, None, None, None], -math.inf)
    e = torch.exp(x - x.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _plain_attention(st, share):
    return torch.matmul(share, _rows_of(st["v_pool"], st["table"])).flatten(2, 3)


def _plain_weighed(st):
    case, table, page = st["case"], st["table"], st["case"]["page"]
    share = _plain_shares(st)
    gathered = st["weights"][:, table.clamp(min=0).long()].permute(1, 0, 3, 2, 4).flatten(3)   # sequence, layer, head, row
    row = torch.arange(table.shape[1] * page, device=DEV)
    fresh = row[None] >= (st["lengths"] - st["counts"])[:, None]
    gathered = torch.where(fresh[:, None, None], 0.0, case["decay"] * gathered) + share.sum(dim=3)
    seq, r = _valid(st).nonzero(as_tuple=True)
    st["weights"][:, table[seq, r // page].long(), :, r % page] = gathered[seq, :, :, r]
    return {"out": _plain_attention(st, share), "weights": st["weights"]}


def _plain_evict(st):
    case, table = st["case"], st["table"]
    n, nl, hkv, page, keep = (case[x] for x in ("n_seq", "layers", "kv_heads", "page", "keep"))
    length = st["lengths"][:, None, None, None]
    w = st["weights"][:, table.clamp(min=0).long()].permute(1, 0, 3, 2, 4).flatten(3)          # sequence, layer, head, row
    i = torch.arange(w.shape[3], device=DEV)
    w = w.masked_fill((i < case["first"]) | (i >= length - case["last"]), math.inf).masked_fill(i >= length, -math.inf)
    rows = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    rows = rows.masked_fill(rows >= length, w.shape[3]).sort(dim=-1).values
    if rows.shape[3] < keep:
        rows = torch.cat([rows, rows.new_full(rows.shape[:3] + (keep - rows.shape[3],), w.shape[3])], dim=3)
    held = rows < w.shape[3]
    seq, layer, head, j = held.nonzero(as_tuple=True)
    r = rows[seq, layer, head, j]
    source, dest = table[seq, r // page].long(), st["after"][seq, j // page].long()
    for pool in ("k_pool", "v_pool", "weights"):
        st[pool][layer, dest, head, j % page] = st[pool][layer, source, head, r % page]
    st["len_out"].copy_(st["lengths"].clamp(max=keep))
    _write_bounds(st, _bounds_of(st, torch.float32, "after", "len_out"), st["after"], st["after"] >= 0)
    st["rows_out"].copy_(rows.masked_fill(~held, -1).view(n * nl * hkv, keep))
    return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "weights": st["weights"], "bounds": st["bounds"], "lengths": st["len_out"], "rows": st["rows_out"]}


def run(state):
    st, case = state, state["case"]
    if not own:
        if case["op"] == "prefix":
            return {"out": _plain_attention(st, _plain_shares(st))}
        return {"normed": _plain_normed, "weighed": _plain_weighed, "evict": _plain_evict}[case["op"]](st)
    from paper_2510_22556_amd import binding as B

    pages, table = st["pages"], st["table"]
    if case["op"] == "normed":
        B.sablock_append_normed_paged(pages, st["tokens"], st["norms"], st["k"], st["v"], st["positions"], st["inv_freq"], table, st["lengths"], st["k_pool"],
                                      st["v_pool"], q=st["q"], q_out=st["q_out"], q_weight=st["q_weight"], k_weight=st["k_weight"], counts=st["counts"],
                                      bounds=st["bounds"])
        return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"], "bounds": st["bounds"]}
    if case["op"] == "weighed":
        B.sablock_decode_weighed_paged(pages, st["q"], st["k_pool"], st["v_pool"], table, st["lengths"], st["weights"], st["out"], st["ws"],
                                       n_new=case["fresh"], counts=st["counts"], decay=case["decay"])
        return {"out": st["out"], "weights": st["weights"]}
    if case["op"] == "evict":
        B.sablock_evict_paged(pages, table, st["lengths"], st["weights"], st["k_pool"], st["v_pool"], case["keep"], st["after"], st["len_out"],
                              st["rows_out"], st["ws"], n_first=case["first"], n_last=case["last"], bounds=st["bounds"])
        return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "weights": st["weights"], "bounds": st["bounds"], "lengths": st["len_out"], "rows": st["rows_out"]}
    B.sablock_decode_prefix_paged(pages, st["q"], st["k_pool"], st["v_pool"], table, st["lengths"], st["begin"], st["prefix_pages"], st["out"], st["ws"])
    return {"out": st["out"]}


# ---- the definitions in 64 bits, one sequence at a time ------------------------------------------------------------------


def _exact_normed(case, st):
    if case["n_seq"] * case["layers"] * case["n_new"] > 2 ** 17:
        return None
    page, R, D = case["page"], case["rotary"], case["dim"]
    kp, vp, bounds, q_out = (st[x].double() for x in ("k_pool", "v_pool", "bounds", "q_out"))
    table = st["table"].tolist()
    for s, (rows, count) in enumerate(zip(_lengths(case), _counts(case))):
        first = rows - count
        place = torch.arange(count, device=DEV, dtype=torch.float64) + float(st["positions"][s])
        done = []
        for x, weight in ((st["k"], st["k_weight"]), (st["q"], st["q_weight"])):
            x, weight = x[s, :, :, :count].double(), weight.double()
            length = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
            x = x / torch.sqrt(length * length / D + EPS) * (weight.unsqueeze(2) if case["per_head"] else weight.unsqueeze(1).unsqueeze(2))
            for i in range(R // 2):
                a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
                # a pair as a complex number, turned by the angle
                z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(place), place * float(st["inv_freq"][i]))
                x[..., a], x[..., b] = z.real, z.imag
            done.append(x)
        q_out[s, :, :, :count] = done[1]
        for r0 in range(first // page * page, rows, page):
            at, lo, hi = table[s][r0 // page], max(first, r0), min(rows, r0 + page)
            kp[:, at, :, lo - r0: hi - r0] = done[0][:, :, lo - first: hi - first]
            vp[:, at, :, lo - r0: hi - r0] = st["v"][s, :, :, lo - first: hi - first].double()
            held = kp[:, at, :, : hi - r0]
            bounds[:, at, :, 0], bounds[:, at, :, 1] = held.amin(dim=2), held.amax(dim=2)
    return {"q": q_out, "k_pool": kp, "v_pool": vp, "bounds": bounds}


def _exact_evict(case, st):
    n, nl, hkv, page, keep = (case[x] for x in ("n_seq", "layers", "kv_heads", "page", "keep"))
    if n * nl * hkv > 1200 or n * nl * hkv * case["rows"] > 2 ** 21:
        return None
    kp, vp, wp, bounds = (st[x].double() for x in ("k_pool", "v_pool", "weights", "bounds"))
    source_w = st["weights"].cpu().numpy()
    table, after, chosen = st["table"].cpu(), st["after"].cpu(), []
    for s, rows in enumerate(_lengths(case)):
        ids = table[s][torch.arange(rows) // page].numpy()
        at = (torch.arange(rows) % page).numpy()
        for l in range(nl):
            for h in range(hkv):
                w = source_w[l, ids, h, at].tolist()
                if rows <= keep:
                    got = list(range(rows))
                else:
                    forced = set(range(case["first"])) | set(range(rows - case["last"], rows))
                    rest = sorted((i for i in range(rows) if i not in forced), key=lambda i: (-w[i], i))
                    got = sorted(list(forced) + rest[: keep - len(forced)])
                chosen.append(got + [-1] * (keep - len(got)))
                src = torch.tensor(got)
                j = torch.arange(len(got))
                a, b = table[s][src // page].long().to(DEV), (src % page).to(DEV)
                c, d = after[s][j // page].long().to(DEV), (j % page).to(DEV)
                for x in (kp, vp, wp):
                    x[l, c, h, d] = x[l, a, h, b]
        for i in range(-(-min(rows, keep) // page)):
            held = kp[:, int(after[s, i]), :, : min(page, min(rows, keep) - i * page)]
            bounds[:, int(after[s, i]), :, 0], bounds[:, int(after[s, i]), :, 1] = held.amin(dim=2), held.amax(dim=2)
    return {"k_pool": kp, "v_pool": vp, "weights": wp, "bounds": bounds, "lengths": _int32([min(r, keep) for r in _lengths(case)]), "rows": _int32(chosen)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "normed":
        return _exact_normed(case, st)
    if case["op"] == "evict":
        return _exact_evict(case, st)
    nl, hkv, page = (case[x] for x in ("layers", "kv_heads", "page"))
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    gathered = st["weights"].double() if case["op"] == "weighed" else None
    for s, rows in enumerate(_lengths(case)):
        r = torch.arange(rows, device=DEV)
        ids, at = st["table"][s].long()[r // page], r % page
        for l in range(nl):
            for h in range(hkv):
                k, v = (st[p][l, ids, h, at].double() for p in ("k_pool", "v_pool"))
                q = st["q"][s, l].view(hkv, -1, case["dim"])[h].double()
                share = torch.softmax((q @ k.t().contiguous()) * case["dim"] ** -0.5, dim=-1)
                out[s, l, h * q.shape[0]: (h + 1) * q.shape[0]] = share @ v
                if gathered is not None:
                    old = gathered[l, ids, h, at] * case["decay"]
                    old[rows - min(case["fresh"], rows):] = 0
                    gathered[l, ids, h, at] = old + share.sum(dim=0)
    return {"out": out} if gathered is None else {"out": out, "weights": gathered}


# ---- what the calls cannot do without -----------------------------------------------------------------------------------


def work(case):
    elt = 4 if case["dtype"] == "f32" else 2
    n, nl, hq, hkv, D, page = (case[x] for x in ("n_seq", "layers", "q_heads", "kv_heads", "dim", "page"))
    lengths = _lengths(case)
    pages = [-(-r // page) for r in lengths]
    row = nl * hkv * D * elt                                             # bytes of K of one row of all problems of a sequence
    if case["op"] == "normed":
        counts = _counts(case)
        touched = sum(-(-r // page) - (r - c) // page for r, c in zip(lengths, counts))
        merged = sum((r - c) % page > 0 for r, c in zip(lengths, counts))                  # pages whose bounds are read as well
        tokens = sum(counts)
        weights = nl * D * ((hq + hkv) if case["per_head"] else 2)
        return {"bytes": tokens * (4 * row + 2 * nl * hq * D * elt) + 2 * row * (touched + merged) + 4 * weights + 4 * touched + 12 * n,
                "flops": tokens * nl * (hq + hkv) * (3.0 * case["rotary"] + 4.0 * D) + 2.0 * tokens * nl * hkv * D}
    if case["op"] == "evict":
        kept = [min(r, case["keep"]) for r in lengths]
        moved = sum(kept)
        return {"bytes": 4 * row * moved + 4 * nl * hkv * (sum(lengths) + 2 * moved) + 2 * row * sum(-(-r // page) for r in kept) + 4 * sum(pages) + 8 * n,
                "flops": 2.0 * nl * hkv * D * moved + nl * hkv * sum(lengths)}
    q = n * nl * hq * D * (elt + 4)
    if case["op"] == "weighed":
        fresh = sum(min(case["fresh"], r) for r in lengths)
        return {"bytes": 2 * row * sum(lengths) + 4 * nl * hkv * (2 * sum(lengths) - fresh) + q + 4 * sum(pages) + 8 * n,
                "flops": nl * hq * (4.0 * D + 1) * sum(lengths)}
    begin, of_prefix = _groups(case)
    own_rows = sum(lengths) - sum(page * m for m in _prefix_pages(case))
    return {"bytes": 2 * row * (own_rows + page * sum(of_prefix)) + q + 4 * (sum(pages) - sum(_prefix_pages(case)) + sum(of_prefix)) + 4 * n + 8 * len(of_prefix),
            "flops": 4.0 * nl * hq * D * sum(lengths)}

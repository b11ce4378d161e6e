"""How a decode step over pages deals out its problems, as the launch and the kernel decide it: for the tests that want a particular way."""


def launch(dtype, D, P, cus, capacity):
    """Workgroups that share the long problems, rows of the longest that one takes alone, rows of a step; no workgroups: every problem is one's."""
    elt = 2 if dtype == "bf16" else 4
    workgroups = min(cus * (3 if D <= 64 else 2 if dtype == "bf16" or D <= 160 else 1), 1023)
    rows_alone = (2 ** 19 if P >= cus else 2 ** 18) // (2 * D * elt)
    alone = capacity <= rows_alone or P * (capacity // 16 + 1) >= 2 ** 30
    return 0 if alone else workgroups, rows_alone, 32 if dtype == "bf16" and D <= 128 and not (alone and D > 64) else 16


def way(dtype, D, page, heads, lengths, max_pages, cus, n_listed=None):
    """alone: a workgroup per problem; short: no long problem among those that may be; cut: runs end with the problems; longer: so do somewhat longer ones;
    even: a workgroup may have pieces of several problems."""
    most = max_pages if n_listed is None else min(n_listed, max_pages)
    workgroups, rows_alone, step = launch(dtype, D, len(lengths) * heads, cus, most * page)
    if not workgroups:
        return "alone"
    up = lambda a, b: -(-a // b)  # noqa: E731
    rows = [min(n, max_pages * page) if n_listed is None else min(n_listed, up(n, page)) * page for n in lengths]
    steps = [n for n in (up(r, step) for r in rows) if n > up(rows_alone, step)]
    if not steps:
        return "short"
    total, problems = sum(steps) * heads, len(steps) * heads
    even = max(4, up(total, workgroups))
    pieces = lambda run: sum(up(n, run) for n in steps) * heads  # noqa: E731
    if pieces(even) <= workgroups:
        return "cut"
    if problems < workgroups:
        run = max(even, up(total, workgroups - problems))
        if run <= even + 4 and pieces(run) <= workgroups:
            return "longer"
    return "even"

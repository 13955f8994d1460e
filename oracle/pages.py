"""Oracle of page admission and release: plain loops over sequences, tokens and pages, as the header words them."""


def extend(table, page_size, lens, new, free, n_free, max_tokens):
    """Lists in, lists out: (table, slots, positions, cu, lens, n_free)."""
    table, lens = [list(r) for r in table], list(lens)
    n0 = min(max(n_free, 0), len(free))
    room = len(table[0]) * page_size if table else 0
    cu, pages, tokens, handed = [0], 0, 0, 0
    slots, positions = [-1] * max_tokens, [0] * max_tokens
    for b, raw in enumerate(new):
        fresh, old = max(raw, 0), max(lens[b], 0)
        cu.append(min(cu[-1] + fresh, 2**31 - 1))
        first, tokens = tokens, tokens + fresh
        if fresh and old + fresh > room:
            continue
        held = -(-old // page_size)
        need = -(-(old + fresh) // page_size) - held if fresh else 0
        pages += need
        if pages > n0 or tokens > max_tokens or not fresh:
            continue
        for c in range(held, held + need):
            table[b][c] = free[n0 - 1 - handed]
            handed += 1
        for t in range(fresh):
            p = old + t
            page = table[b][p // page_size]
            positions[first + t] = p
            slots[first + t] = page * page_size + p % page_size if page >= 0 else -1
        lens[b] = old + fresh
    return table, slots, positions, cu, lens, n0 - handed


def release(table, page_size, lens, keep, free, n_free):
    """(free pages, lens, n_free)."""
    free, lens = list(free), list(lens)
    n = min(max(n_free, 0), len(free))
    for b, want in enumerate(keep):
        old = lens[b]
        lens[b] = min(old, max(want, 0))
        for c in range(-(-max(lens[b], 0) // page_size), min(-(-max(old, 0) // page_size), len(table[b]))):
            if n < len(free):
                free[n] = table[b][c]
                n += 1
    return free, lens, n

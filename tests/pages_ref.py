"""What the page calls compute, one slot and one page at a time in plain Python."""
PAGE = 16


def pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def update(table, lens, refs, new_lens, parent=None):
    """Lists in, lists out: table, lens, refs, pages left, copies [(from, to)].  Not enough pages: the inputs and no copies."""
    B, P = len(lens), len(refs)
    parent = list(range(B)) if parent is None else parent
    out, count = [[-1] * len(table[0]) for _ in range(B)], list(refs)
    is_page = lambda e: 0 <= e < P  # noqa: E731
    for r in range(B):
        for e in table[r][:pages(lens[r])]:
            if is_page(e):
                count[e] -= 1
    keep = [0 if s < 0 else min(lens[s], n) for s, n in zip(parent, new_lens)]
    for r in range(B):
        for b in range(pages(keep[r])):
            out[r][b] = table[parent[r]][b]
            if is_page(out[r][b]):
                count[out[r][b]] += 1
    open_on = {}                                                    # page -> rows that end inside it
    for r in range(B):
        if keep[r] % PAGE and is_page(out[r][keep[r] // PAGE]):
            open_on.setdefault(out[r][keep[r] // PAGE], []).append(r)
    copied = set()
    for e, rows in open_on.items():
        copied |= set(rows if count[e] > len(rows) else rows[1:])
    free = [e for e in range(P) if count[e] == 0]
    wanted = [(r, b) for r in range(B) for b in ([keep[r] // PAGE] if r in copied else []) + list(range(pages(keep[r]), pages(new_lens[r])))]
    if len(wanted) > len(free):
        return [list(t) for t in table], list(lens), list(refs), len(free) - len(wanted), []
    copies = []
    for (r, b), e in zip(wanted, free):
        if r in copied and b == keep[r] // PAGE:
            copies.append((out[r][b], e))
            count[out[r][b]] -= 1
        out[r][b] = e
        count[e] += 1
    return out, list(new_lens), count, len(free) - len(wanted), copies


def compact(table, lens, refs):
    """table, refs, map, live pages, moves [(from, to)]."""
    n = sum(c > 0 for c in refs)
    moves = list(zip([e for e in range(n, len(refs)) if refs[e] > 0], [e for e in range(n) if refs[e] <= 0]))
    where = {e: e for e in range(len(refs)) if refs[e] > 0}
    where.update(moves)
    out = [[where.get(e, e) if b < pages(t) and e >= 0 else e for b, e in enumerate(row)] for row, t in zip(table, lens)]
    count = [0] * len(refs)
    for e, f in where.items():
        count[f] = refs[e]
    return out, count, [where.get(e, -1) for e in range(len(refs))], n, moves

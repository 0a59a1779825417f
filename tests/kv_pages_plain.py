"""Page tables whose rows share pages, from their definition: lists and loops.  table: rows of page numbers; refs: entries that name each page."""


def count(table, pages):
    refs = [0] * pages
    for row in table:
        for p in row:
            if 0 <= p < pages:
                refs[p] += 1
    return refs


def fork(table, pages, P, src, length=None):
    """The new table (an entry that is no page is -1 where it is taken over)."""
    wide, new = len(table[0]), []
    for b, s in enumerate(src):
        keep = 0
        if 0 <= s < len(table):
            keep = wide if length is None else min(-(-max(int(length[b]), 0) // P), wide)
        row = [p if 0 <= p < pages else -1 for p in table[s][:keep]] if keep else []
        new.append(row + [-1] * (wide - keep))
    return new


def reserve(table, refs, P, start, n):
    """Changes table and refs.  Returns (missing, copies (from, to), wiped: new pages that hold nothing)."""
    pages, wide = len(refs), len(table[0])
    before, free = list(refs), [p for p, r in enumerate(refs) if r == 0]
    missing, copies, wiped, r = [0] * len(table), [], [], 0
    for b, row in enumerate(table):
        if start[b] < 0 or n[b] <= 0:
            continue
        for j in range(start[b] // P, min((start[b] + n[b] - 1) // P + 1, wide)):
            p = row[j]
            held = 0 <= p < pages
            if held and before[p] <= 1:
                continue
            if r == len(free):
                missing[b] += 1
                continue
            if held:
                refs[p] -= 1
            (copies if held and j * P < start[b] else wiped).append((p, free[r]))
            row[j] = free[r]
            refs[free[r]] = 1
            r += 1
    return missing, copies, [q for _, q in wiped]


def compact(table, refs):
    """Changes table and refs.  Returns (used, moved, moves (from, to))."""
    used = sum(r > 0 for r in refs)
    moves = list(zip([p for p in range(used, len(refs)) if refs[p] > 0], [p for p in range(used) if refs[p] <= 0]))
    moved = [p if r > 0 else -1 for p, r in enumerate(refs)]
    for a, b in moves:
        moved[a] = b
        refs[a], refs[b] = 0, refs[a]
    for row in table:
        for j, p in enumerate(row):
            if 0 <= p < len(refs):
                row[j] = moved[p]
    return used, moved, moves

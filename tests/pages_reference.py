"""Plain statements, on lists, of what the calls of include/sssd_kv8.h do to a pool's table, counts and pages: one slot after the other.  Each
returns None where it has to do nothing, else the new state and the pages that are copied (from, to)."""
BLOCK = 32


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def sound(table, refs):
    return all(-1 <= p < len(refs) and (p < 0 or refs[p] > 0) for row in table for p in row)


def fork(table, refs, lens, origins, max_seq):
    slots, per = len(table), len(table[0])
    if any(o < -1 or o >= slots for o in origins) or not sound(table, refs):
        return None
    if any(o >= 0 and not 0 <= lens[o] <= max_seq for o in origins):
        return None
    length = [lens[o] if o >= 0 else 0 for o in origins]
    if any(o >= 0 and -1 in table[o][:blocks(n)] for o, n in zip(origins, length)):
        return None
    new, asks = [], []
    for b, (o, n) in enumerate(zip(origins, length)):
        row = [table[o][i] if i < blocks(n) else -1 for i in range(per)]
        if n % BLOCK:
            heir = o if origins[o] == o else origins.index(o)
            if heir != b:
                asks.append((b, n // BLOCK, row[n // BLOCK]))
                row[n // BLOCK] = -1
        new.append(row)
    counts = list(refs)
    for was, now in zip(table, new):
        for p, q in zip(was, now):
            if p >= 0:
                counts[p] -= 1
            if q >= 0:
                counts[q] += 1
    free = [p for p, n in enumerate(counts) if n == 0]
    if len(free) < len(asks):
        return None
    copies = []
    for (b, i, page), to in zip(asks, free):
        new[b][i] = to
        counts[to] = 1
        copies.append((page, to))
    return new, counts, length, copies


def reserve(table, refs, lens, counts, first, n, max_seq):
    if any(a < 0 or c < 0 or c > n or a + c > max_seq for a, c in zip(lens, counts)):
        return None
    asks = [(first + k, i, a) for k, (a, c) in enumerate(zip(lens, counts)) if c for i in range(a // BLOCK, blocks(a + c))]
    if not sound([[table[b][i] for b, i, _ in asks]], refs):
        return None
    of = {}
    for b, i, _ in asks:
        of.setdefault(table[b][i], []).append((b, i))
    new, now, wants = [list(r) for r in table], list(refs), []
    for b, i, a in asks:
        p = table[b][i]
        if p < 0 or (refs[p] > 1 and not (len(of[p]) == refs[p] and of[p][0] == (b, i))):
            wants.append((b, i, p, a))
    free = [p for p, c in enumerate(refs) if c == 0]
    if len(free) < len(wants):
        return None
    copies = []
    for (b, i, p, a), to in zip(wants, free):
        new[b][i] = to
        now[to] = 1
        if p >= 0:
            now[p] -= 1
            if i * BLOCK < a:
                copies.append((p, to))
    return new, now, copies


def compact(table, refs, to_pages=None):
    """-> (table, counts, where each page is, copies, pages in use)."""
    used = [p for p, n in enumerate(refs) if n > 0]
    if not sound(table, refs) or (to_pages is not None and len(used) > to_pages):
        return None
    if to_pages is None:
        copies = list(zip([p for p in used if p >= len(used)], [p for p in range(len(used)) if refs[p] <= 0]))
        where = {p: p for p in used}
        where.update(copies)
        counts = [0] * len(refs)
    else:
        where = {p: i for i, p in enumerate(used)}
        copies = list(where.items())
        counts = [0] * to_pages
    for p in used:
        counts[where[p]] = refs[p]
    return [[where[p] if p >= 0 else -1 for p in row] for row in table], counts, [where.get(p, -1) for p in range(len(refs))], copies, len(used)

"""The upkeep of a paged cache, entry by entry on plain lists: what the device
operators are compared with.  Values are integers; a cache is a NumPy array
[pages, kv heads, page size, head dim]."""

from __future__ import annotations


def pages_of(tokens, page):
    return -(-max(tokens, 0) // page)


def lowest_free(refs, count):
    return [p for p, r in enumerate(refs) if r <= 0][:count]


def append(k, v, k_cache, v_cache, table, lens, starts, page):
    pages = k_cache.shape[0]
    for s, n in enumerate(lens):
        first, end = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
        for row in range(first, end):
            place = n - (end - row)
            if place < 0 or place // page >= len(table[s]):
                continue
            p = table[s][place // page]
            if 0 <= p < pages:
                k_cache[p, :, place % page] = k[row]
                v_cache[p, :, place % page] = v[row]


def reserve(table, refs, old, new, page):
    """The shortfall; table and refs change only when it is 0."""
    width = len(table[0])
    wanted = [(s, e) for s in range(len(table)) for e in range(min(pages_of(old[s], page), width), min(pages_of(new[s], page), width))
              if table[s][e] < 0]
    free = lowest_free(refs, len(wanted))
    if len(free) < len(wanted):
        return len(wanted) - len(free)
    for (s, e), p in zip(wanted, free):
        table[s][e] = p
        refs[p] = 1
    return 0


def free(table, refs, lens, seqs, page, window=0, sinks=0):
    for s in seqs:
        if not 0 <= s < len(table):
            continue
        for e, p in enumerate(table[s]):
            kept = any(t < sinks or (window > 0 and t + window > lens[s]) for t in range(e * page, e * page + page))
            if p < 0 or kept:
                continue
            table[s][e] = -1
            if p < len(refs):
                refs[p] -= 1


def fork(caches, table, refs, lens, src, dst, page):
    width, jobs = len(table[0]), []
    for s, d in zip(src, dst):
        if not (0 <= s < len(table) and 0 <= d < len(table)) or not 0 <= lens[s] <= width * page:
            continue
        full, part = divmod(lens[s], page)
        jobs.append((s, d, full, part, part > 0 and 0 <= table[s][full] < len(refs)))
    want = sum(j[4] for j in jobs)
    free_pages = lowest_free(refs, want)
    if len(free_pages) < want:
        return want - len(free_pages)
    for s, d, full, part, own in jobs:
        row = [table[s][e] if e < full else -1 for e in range(width)]
        for p in row:
            if 0 <= p < len(refs):
                refs[p] += 1
        if own:
            row[full] = free_pages.pop(0)
            refs[row[full]] = 1
            for c in caches:
                c[row[full], :, :part] = c[table[s][full], :, :part]
        table[d] = row
        lens[d] = lens[s]
    return 0


def compact(caches, table, refs):
    """(new table, new refs, pages in use)."""
    live = [p for p, r in enumerate(refs) if r > 0]
    n = len(live)
    move = dict(zip([p for p in live if p >= n], [p for p in range(n) if refs[p] <= 0]))
    for a, b in move.items():
        for c in caches:
            c[b] = c[a]
    new_refs = [refs[p] if refs[p] > 0 and p < n else 0 for p in range(len(refs))]
    for a, b in move.items():
        new_refs[b] = refs[a]
    return [[move.get(p, p) for p in row] for row in table], new_refs, n

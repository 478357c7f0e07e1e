"""Plain statements of the operators for requests that share prefixes, sequence by sequence in Python lists (test infrastructure)."""


def admit(table, lens, refs, like, begin, total, page):
    width, old = len(table[0]), (table, lens, refs)
    refs, new, keeps = list(refs), [], []
    for i, p in enumerate(like):
        k = min(begin[i], lens[p], total[i]) if p >= 0 else 0
        if not (p == i and k == lens[i]):
            k -= k % page
        n = -(-k // page)
        new.append((list(table[p][:n]) if p >= 0 else []) + [-1] * (width - n))
        keeps.append(k)
    for row in new:
        for x in row:
            if x >= 0:
                refs[x] += 1
    for row, n in zip(table, lens):
        for x in row[: -(-n // page)]:
            if x >= 0:
                refs[x] -= 1
    if any(t > width * page for t in total):
        return *old, [0] * len(lens), -4
    want = [(i, j) for i, k in enumerate(keeps) for j in range(-(-k // page), -(-total[i] // page))]
    free = [x for x, r in enumerate(refs) if r == 0]
    if len(want) > len(free):
        return *old, [0] * len(lens), -4
    for (i, j), x in zip(want, free):
        new[i][j] = x
        refs[x] = 1
    return new, list(total), refs, [t - k for t, k in zip(total, keeps)], 0


def slots(table, lens, n_new, page, rows):
    q_start, positions, seqs, slot = [0], [], [], []
    for s, n in enumerate(n_new):
        q_start.append(q_start[-1] + n)
        for p in range(lens[s] - n, lens[s]):
            positions.append(p)
            seqs.append(s)
            slot.append(table[s][p // page] * page + p % page)
    pad = [-1] * (rows - q_start[-1])
    return q_start, positions + pad, seqs + pad, slot + pad


def groups(table, lens, q_start, page, least):
    lead, shared = [], []
    whole = [max(0, n - (q_start[s + 1] - q_start[s])) // page for s, n in enumerate(lens)]
    for s in range(len(lens)):
        c = 0
        while s and c < min(whole[s - 1], whole[s], len(table[0])) and table[s][c] == table[s - 1][c] and table[s][c] >= 0:
            c += 1
        linked = c > 0 and c * page >= least
        lead.append(lead[-1] if linked else s)
        shared.append(c if linked else None)
    of = {}
    for l, c in zip(lead, shared):
        if c is not None:
            of[l] = min(of.get(l, c), c)
    return lead, [of.get(l, 0) * page for l in lead]

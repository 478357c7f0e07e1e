"""Plain 64-bit statements of the operators on a paged cache, and builders of their inputs (test infrastructure).

The pages' bookkeeping is stated sequence by sequence in Python; attention and rotary positions in float64 torch, dense, one sequence and
head group at a time.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # unit roundoff
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half the smallest subnormal


def rope(x, positions, inv_freq, interleaved, scale):
    """x [tokens, heads, dh] -> float64, turned."""
    x = x.double().clone()
    r = 2 * inv_freq.numel()
    a = positions.clamp(min=0).double()[:, None, None] * inv_freq.double()
    i0, i1 = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    x0, x1 = x[..., i0].clone(), x[..., i1].clone()
    x[..., i0] = scale * (x0 * a.cos() - x1 * a.sin())
    x[..., i1] = scale * (x1 * a.cos() + x0 * a.sin())
    return x


def cache(lens, page, hkv, dh, dtype, seed, *, layers=1, layer=1, spare=3, width=None, fill=float("nan"), device="cuda"):
    """A pool filled with `fill`, the sequences' pages in random places, normal K and V in positions 0 .. lens - 1 of block `layer`."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    width = width or max(1, max(need) + 1)
    n_pages = sum(need) + spare
    ids = torch.randperm(n_pages, generator=g)
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    pool = torch.full((layers, n_pages, 2, hkv, page, dh), fill, dtype=dtype)
    for s, n in enumerate(lens):
        for j in range(need[s]):
            table[s, j] = ids[at]
            m = min(page, n - j * page)
            pool[layer - 1, ids[at], :, :, :m] = torch.randn(2, hkv, m, dh, generator=g).to(dtype)
            at += 1
    return pool.to(device), table.to(device), torch.tensor(lens, dtype=torch.int32, device=device)


def sequence(pool, layer, table, s, n):
    """K, V of positions 0 .. n - 1 of sequence s: [n, Hkv, dh] each."""
    page = pool.shape[4]
    j = torch.arange(n, device=pool.device)
    kv = pool[layer - 1, table[s].long()[j // page], :, :, j % page]
    return kv[:, 0], kv[:, 1]


def visible(n, new, window, sinks, device):
    """[new, n]: which positions the last `new` queries of a sequence of n positions see."""
    p, j = torch.arange(n - new, n, device=device)[:, None], torch.arange(n, device=device)
    return (j <= p) & ((j < sinks) | (j > p - window))


def attention(q, starts, pool, layer, table, lens, window, sinks, scale):
    """-> (float64 result, bound): the bound covers one rounding of the result, one of every probability (relative to sum p |v|), and the
    fp32 arithmetic of scores (dh + 4 roundings of products and sums), exponentials and sums; see the terms."""
    t, hq, dh = q.shape
    g = hq // pool.shape[3]
    out = torch.zeros(t, hq, dh, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    u = U[q.dtype]
    for s, n in enumerate(lens):
        a, b = starts[s], starts[s + 1]
        if b == a or n <= 0:
            continue
        first = max(0, b - a - n)  # queries before position 0 see nothing
        m = visible(n, b - a - first, window, sinks, q.device)
        need = m.any(0).nonzero().flatten()
        page = pool.shape[4]
        kv = pool[layer - 1, table[s].long()[need // page], :, :, need % page].double()
        m = m[:, need]
        for h in range(hq):
            x, k, v = q[a + first:b, h].double(), kv[:, 0, h // g], kv[:, 1, h // g]
            sc = (x @ k.T * scale).masked_fill(~m, -math.inf)
            p = torch.softmax(sc, -1)
            out[a + first:b, h] = p @ v
            mass = p @ v.abs()
            spread = (x.abs() @ k.abs().T * abs(scale)).masked_fill(~m, 0).amax(-1, keepdim=True)
            fp32 = 2 * (dh + 8) * 2.0 ** -24 * spread + (len(need) + 8) * 2.0 ** -23
            tol[a + first:b, h] = u * out[a + first:b, h].abs() + (u + fp32) * mass * (1 + u) + len(need) * TINY[q.dtype] * v.abs().max() + TINY[q.dtype]
    return out, tol


# ---------------------------------------------------------------- pages, in Python lists
def free_ids(refs):
    return [p for p, r in enumerate(refs) if r == 0]


def advance(table, lens, refs, n_new, page, window, sinks):
    table, lens, refs = [list(r) for r in table], list(lens), list(refs)
    width = len(table[0])
    for s, row in enumerate(table):
        if window > 0:
            j = min((lens[s] - window + 1) // page, width) - 1
            while j >= -(-sinks // page) and row[j] >= 0:
                refs[row[j]] -= 1
                row[j] = -1
                j -= 1
    want = [(s, j) for s in range(len(lens)) for j in range(-(-lens[s] // page), -(-(lens[s] + n_new[s]) // page))]
    free = free_ids(refs)
    if len(want) > len(free) or any(n + m > width * page for n, m in zip(lens, n_new)):
        return table, lens, refs, -4
    for (s, j), p in zip(want, free):
        table[s][j] = p
        refs[p] = 1
    return table, [n + m for n, m in zip(lens, n_new)], refs, 0


def reorder(table, lens, refs, parents, page):
    old_table, old_lens, old_refs = table, lens, refs
    refs, width = list(refs), len(table[0])
    held = lambda s: [p for p in old_table[s][: -(-old_lens[s] // page)] if p >= 0]  # noqa: E731
    new, new_lens, wants, seen = [], [], [], set()
    for i, p in enumerate(parents):
        row, n = [-1] * width, 0
        if p >= 0:
            n = old_lens[p]
            for j in range(-(-n // page)):
                row[j] = old_table[p][j]
            if n % page and p in seen and row[n // page] >= 0:
                wants.append((i, n // page, row[n // page], n % page))
                row[n // page] = -1
            seen.add(p)
        new.append(row)
        new_lens.append(n)
    for row in new:
        for x in row:
            if x >= 0:
                refs[x] += 1
    for s in range(len(old_lens)):
        for x in held(s):
            refs[x] -= 1
    free = free_ids(refs)
    if len(wants) > len(free):
        return old_table, old_lens, old_refs, [], -4
    copies = []
    for (i, j, src, fill), dst in zip(wants, free):
        new[i][j] = dst
        refs[dst] = 1
        copies.append((src, dst, fill))
    return new, new_lens, refs, copies, 0


def compact(table, refs):
    used = [p for p, r in enumerate(refs) if r > 0]
    n = len(used)
    movers, holes = [p for p in used if p >= n], [p for p in range(n) if refs[p] <= 0]
    remap = [p if r > 0 else -1 for p, r in enumerate(refs)]
    refs = list(refs)
    for a, b in zip(movers, holes):
        remap[a] = b
        refs[b], refs[a] = refs[a], 0
    return [[remap[x] if 0 <= x < len(refs) else -1 for x in row] for row in table], refs, remap, n, list(zip(movers, holes))

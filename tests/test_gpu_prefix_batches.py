"""The page tables of requests, the places of new tokens and the groups that share pages, against plain Python (needs a B200).  All of it is exact."""
import random

import pytest
import torch

from paper_2604_18396_b200 import pages_admit, pages_slots, prefix_groups
from tests import prefix_reference as ref

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def state(rng, seqs, width, page, pages, share=0.3):
    """Sequences with pages in random places; some begin with the whole pages of the one before."""
    ids = rng.sample(range(pages), pages)
    table, lens, refs = [], [], [0] * pages
    for s in range(seqs):
        n = rng.choice([0, 1, page, rng.randint(0, width * page)])
        row = [-1] * width
        first = rng.randint(0, min(n, lens[-1]) // page) if s and rng.random() < share else 0
        for j in range(-(-n // page)):
            row[j] = table[-1][j] if j < first else (ids.pop() if ids else -1)
            if row[j] < 0:
                n = j * page
                break
            refs[row[j]] += 1
        table.append(row)
        lens.append(n)
    return table, lens, refs


def run_admit(table, lens, refs, like, begin, total, page, stream=None):
    t, n, r = i32(table), i32(lens), i32(refs)
    outs = [torch.full_like(x, -99) for x in (t, n, r, n)] + [i32([7])]
    pages_admit(t, n, r, i32(like), i32(begin), i32(total), *outs, page_size=page, stream=stream)
    return [x.tolist() for x in outs[:4]] + [outs[4].item()]


@pytest.mark.parametrize("seqs,width,page,pages", [(1, 1, 16, 1), (1, 9, 16, 12), (4, 8, 32, 40), (7, 33, 64, 100), (64, 21, 16, 900), (300, 40, 16, 5000), (1100, 6, 32, 4001),
                                                   (40, 700, 16, 20000), (3, 90000, 16, 270000)])
def test_admit(seqs, width, page, pages):
    rng = random.Random(seqs + width)
    for trial in range(3):
        table, lens, refs = state(rng, seqs, width, page, pages)
        like = [rng.choice([i, i, -1, rng.randrange(seqs)]) for i in range(seqs)]
        begin = [rng.choice([0, lens[p], rng.randint(0, lens[p] + 20)]) if p >= 0 else rng.choice([0, 5]) for p in like]
        total = [min(width * page, rng.choice([0, b, b + 1, b + rng.randint(0, 3 * page)])) for b in begin]
        assert run_admit(table, lens, refs, like, begin, total, page) == list(ref.admit(table, lens, refs, like, begin, total, page))


def test_admit_without_room():
    """Too few pages, a row too short: the state as it was, and no new positions."""
    rng = random.Random(4)
    table, lens, refs = state(rng, 5, 10, 16, 60, share=0)
    for total in ([160, 160, 160, 160, 160], [0, 0, 161, 0, 0], [2 ** 31 - 1] * 5):
        refs2 = [max(r, int(i >= 20)) for i, r in enumerate(refs)]
        got = run_admit(table, lens, refs2, [-1] * 5, [0] * 5, total, 16)
        assert got == [table, lens, refs2, [0] * 5, -4] or sum(-(-t // 16) for t in total) <= sum(r == 0 for r in refs2)


@pytest.mark.parametrize("what,value", [("like", -2), ("like", 5), ("like", 2 ** 31 - 1), ("begin", -1), ("total", -1), ("lens", -1), ("lens", 161), ("table", 60), ("table", 2 ** 30)])
def test_admit_numbers_out_of_range(what, value):
    rng = random.Random(5)
    table, lens, refs = state(rng, 5, 10, 16, 60, share=0)
    lens[2], table[2] = 32, [*[x for x in range(60) if refs[x] == 0][:2], *[-1] * 8]
    a = {"table": table, "lens": lens, "refs": refs, "like": [0, 1, 2, 3, 4], "begin": list(lens), "total": list(lens)}
    if what == "table":
        table[2][1] = value
    else:
        a[what][2] = value
    got = run_admit(**a, page=16)
    assert got == [a["table"], a["lens"], refs, [0] * 5, -1]


@pytest.mark.parametrize("seqs,width,page,most,pad", [(1, 4, 16, 1, 0), (1, 4, 16, 0, 3), (8, 10, 16, 1, 0), (33, 12, 64, 40, 7), (256, 64, 16, 300, 1000), (3000, 5, 32, 3, 1), (2, 3000, 16, 30000, 5)])
def test_slots(seqs, width, page, most, pad):
    rng = random.Random(seqs)
    table = [[rng.randint(0, 2 ** 31 // page * 4) % (2 ** 31 - 1) for _ in range(width)] for _ in range(seqs)]  # (slots beyond 32 bits)
    n_new = [rng.randint(0, min(most, width * page)) for _ in range(seqs)]
    lens = [rng.randint(n, width * page) for n in n_new]
    rows = sum(n_new) + pad
    q_start, positions, sq = i32([5] * (seqs + 1)), i32([5] * rows), i32([5] * rows)
    slots, status = torch.full((rows,), 5, dtype=torch.int64, device="cuda"), i32([0])
    pages_slots(i32(table), i32(lens), i32(n_new), q_start, positions, sq, slots, page_size=page, status=status)
    assert (q_start.tolist(), positions.tolist(), sq.tolist(), slots.tolist()) == ref.slots(table, lens, n_new, page, rows) and status.item() == 0


def test_slots_that_are_none():
    def call(table, lens, n_new, rows):
        o = [i32([5] * (len(lens) + 1)), i32([5] * rows), i32([5] * rows), torch.full((rows,), 5, dtype=torch.int64, device="cuda"), i32([0])]
        pages_slots(i32(table), i32(lens), i32(n_new), *o[:4], page_size=16, status=o[4])
        return [x.tolist() for x in o]

    table = [[3, 4], [5, -1], [6, 7]]
    assert call(table, [17, 17, 2], [1, 2, 0], 3) == [[0, 1, 3, 3], [16, 15, 16], [0, 1, 1], [64, 95, -1], [-1]]          # a page that is missing
    assert call(table, [17, 1, 33], [0, 2, 1], 4) == [[0, 0, 2, 3], [-1, 0, 32, -1], [1, 1, 2, -1], [-1, 80, -1, -1], [-1]]  # before position 0, past the table
    assert call(table, [17, 9, 2], [1, -3, 1], 2) == [[0, 1, 1, 2], [16, 1], [0, 2], [64, 97], [-1]]                      # a negative number
    assert call(table, [17, 9, 2], [2, 0, 1], 2) == [[0, 0, 0, 0], [-1, -1], [-1, -1], [-1, -1], [-1]]                    # more than there are rows
    assert call(table, [17, 9, 2], [2 ** 31 - 1] * 3, 2) == [[0, 0, 0, 0], [-1, -1], [-1, -1], [-1, -1], [-1]]
    assert call(table, [17, 9, 2], [0, 0, 0], 0) == [[0, 0, 0, 0], [], [], [], [0]]


@pytest.mark.parametrize("seqs,width,page", [(1, 1, 16), (2, 5, 16), (9, 40, 32), (40, 300, 16), (70, 400, 64), (1000, 16, 16), (1030, 20, 16), (5000, 37, 16), (12, 5000, 16)])
def test_groups(seqs, width, page):
    rng = random.Random(seqs)
    for least in (1, page + 1, 10 * page):
        table, lens, q_start = [], [], [0]
        for s in range(seqs):
            row = [rng.randint(0, 9999) for _ in range(width)]
            if s and rng.random() < 0.85:
                c = rng.choice([width, rng.randint(0, width), rng.randint(0, min(width, 12))])
                row[:c] = table[-1][:c]
            if rng.random() < 0.1:
                row[rng.randrange(width)] = -1
            table.append(row)
            lens.append(rng.choice([width * page, width * page, rng.randint(0, width * page)]))
            q_start.append(q_start[-1] + rng.choice([0, 1, 1, rng.randint(0, 2 * page), lens[-1] + 1]))
        lead, shared = i32([-5] * seqs), i32([-5] * seqs)
        prefix_groups(i32(table), i32(lens), i32(q_start), lead, shared, page_size=page, least=least)
        assert (lead.tolist(), shared.tolist()) == ref.groups(table, lens, q_start, page, least)


def test_in_a_graph_and_on_another_stream():
    rng = random.Random(9)
    table, lens, refs = state(rng, 40, 300, 16, 9000)
    like = [i if i % 3 else -1 for i in range(40)]
    begin, total = list(lens), [min(4800, n + 20) for n in lens]
    want = list(ref.admit(table, lens, refs, like, begin, total, 16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert run_admit(table, lens, refs, like, begin, total, 16) == want
    t, n, r, args = i32(table), i32(lens), i32(refs), [i32(x) for x in (like, begin, total)]
    outs = [torch.empty_like(x) for x in (t, n, r, n)] + [i32([7])]
    rows = sum(want[3])
    q_start, positions, sq, lead, shared = i32([0] * 41), i32([0] * rows), i32([0] * rows), i32([0] * 40), i32([0] * 40)
    slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages_admit(t, n, r, *args, *outs, page_size=16)
        pages_slots(outs[0], outs[1], outs[3], q_start, positions, sq, slots, page_size=16)
        prefix_groups(outs[0], outs[1], q_start, lead, shared, page_size=16)
    for _ in range(2):
        for x in (*outs, q_start, positions, sq, slots, lead, shared):
            x.fill_(-9)
        graph.replay()
        assert [x.tolist() for x in outs[:4]] + [outs[4].item()] == want
        assert (q_start.tolist(), positions.tolist(), sq.tolist(), slots.tolist()) == ref.slots(want[0], want[1], want[3], 16, rows)
        assert (lead.tolist(), shared.tolist()) == ref.groups(want[0], want[1], q_start.tolist(), 16, 1)

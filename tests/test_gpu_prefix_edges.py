"""Sizes beyond 32 bits, page tables that the other SMs help with, and chains in a graph, for requests that share prefixes (needs a B200).

Tolerances as in the files of the operators: `paged_reference.attention` derives its own, the rest is exact.
"""
import random

import pytest
import torch

from paper_2604_18396_b200 import pages_admit, pages_slots, prefix_attention, prefix_groups
from tests import paged_reference as paged, prefix_reference as ref
from tests.test_gpu_prefix_attention import ALL, BF, GROUPS, NAN, Batch, i32
from tests.test_gpu_prefix_batches import run_admit, state

pytestmark = pytest.mark.gpu


def test_pages_behind_four_gigabytes():
    """The second block of a pool whose blocks are 4.3 GB: rows and bytes of the last pages pass 31 and 32 bits."""
    b = Batch([(256, [(70, 1), (0, 1), (5, 2)]), (64, [(100, 1), (3, 1)])], 16, 8, 128, 64, BF)
    n, far = b.pool.shape[1], 16500
    pool = torch.empty(2, far + n, 2, 8, 64, 128, dtype=BF, device="cuda")
    pool[1, far:] = b.pool[0]
    pool[0, far:] = NAN
    pool[1, :n] = NAN
    b.pool, b.layer = pool, 2
    b.table = torch.where(b.table >= 0, b.table + far, b.table)
    b.check()


def wide(rng, pages):
    """Three sequences whose tables are as wide as the other SMs are called for."""
    return state(rng, 3, 90000, 16, pages, share=1.0)


def test_wide_tables_without_room_and_out_of_range():
    rng = random.Random(11)
    table, lens, refs = wide(rng, 20000)
    free = sum(r == 0 for r in refs)
    for total in ([90000 * 16 + 1, 0, 5], [(free + 60000) * 16, 3, 0]):
        assert run_admit(table, lens, refs, [-1] * 3, [0] * 3, total, 16) == [table, lens, refs, [0] * 3, -4]
    for like in ([3, -1, -1], [0, -2, -1]):
        assert run_admit(table, lens, refs, like, [0] * 3, [16] * 3, 16) == [table, lens, refs, [0] * 3, -1]


@pytest.mark.parametrize("seqs,width,pages", [(5, 40, 300), (3, 90000, 20000)])
def test_admission_replayed_on_other_requests(seqs, width, pages):
    """A captured call reads what its arrays hold when it is replayed."""
    rng = random.Random(seqs)
    table, lens, refs = state(rng, seqs, width, 16, pages)
    arrays = {"like": [-1] * seqs, "begin": [0] * seqs, "total": [1] * seqs}
    t, n, r, dev = i32(table), i32(lens), i32(refs), {k: i32(v) for k, v in arrays.items()}
    outs = [torch.full_like(x, -99) for x in (t, n, r, n)] + [i32([7])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages_admit(t, n, r, dev["like"], dev["begin"], dev["total"], *outs, page_size=16)
    for trial in range(3):
        like = [rng.choice([i, -1, rng.randrange(seqs)]) for i in range(seqs)]
        begin = [lens[p] if p >= 0 else 0 for p in like]
        total = [b + rng.randint(0, 40) if trial < 2 else width * 16 + 1 for b in begin]
        total = [min(x, width * 16) if trial < 2 else x for x in total]
        for k, v in (("like", like), ("begin", begin), ("total", total)):
            dev[k].copy_(i32(v))
        graph.replay()
        assert [x.tolist() for x in outs[:4]] + [outs[4].item()] == list(ref.admit(table, lens, refs, like, begin, total, 16))


def test_everything_in_one_graph_twice():
    """Slots, groups and attention captured together; the last replay has other lengths, other groups and fewer tokens, one before it
    a position without a page."""
    page, hq, hkv, dh, rows = 16, 8, 2, 128, 12
    b = Batch([(640, [(5, 1), (40, 2), (9, 1)]), (96, [(30, 3), (200, 1)])], hq, hkv, dh, page, BF)
    table, lens, n_new = b.table.clone(), b.lens_t.clone(), i32([1, 2, 1, 3, 1])
    q = torch.randn(rows, hq, dh, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    out = torch.full_like(q, 7.0)
    q_start, positions, seqs, lead, shared = (i32([0] * k) for k in (6, rows, rows, 5, 5))
    slots, status = torch.zeros(rows, dtype=torch.int64, device="cuda"), i32([0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages_slots(table, lens, n_new, q_start, positions, seqs, slots, page_size=page, status=status)
        prefix_groups(table, lens, q_start, lead, shared, page_size=page)
        prefix_attention(q, out, q_start, b.pool, 1, table, lens, lead, shared, max_q=3, max_own=250, status=status)
    for new, rest in (([1, 2, 1, 3, 1], b.lens), ([1, 0, 1, 1, 1], [700, 650, 64, 100, 130]), ([1, 0, 1, 1, 1], [600, 650, 64, 100, 130])):
        lens.copy_(i32(rest))
        n_new.copy_(i32(new))
        out.fill_(7.0)
        graph.replay()
        t = sum(new)
        if rest[0] == 700:  # (the first sequence has pages for 656 positions)
            assert status.item() == -1 and slots[0].item() == -1
            status.zero_()
            continue
        assert status.item() == 0
        assert (q_start.tolist(), positions.tolist(), seqs.tolist(), slots.tolist()) == ref.slots(table.tolist(), rest, new, page, rows)
        assert (lead.tolist(), shared.tolist()) == ref.groups(table.tolist(), rest, q_start.tolist(), page, 1)
        want, tol = paged.attention(q[:t], q_start.tolist(), b.pool, 1, table, rest, ALL, 0, dh ** -0.5)
        assert ((out[:t].double() - want).abs() <= tol).all() and (out[t:] == 7.0).all()


def test_one_sequence_and_one_page_table_entry():
    """The smallest calls there are."""
    for n, new in ((1, 1), (16, 1), (16, 16), (9, 4)):
        b = Batch([(0, [(n - new, new)])], 2, 1, 64, 16, BF)
        b.table = b.table[:, :1].contiguous()
        b.check()


def test_the_same_sequence_twice_in_a_batch():
    """Two rows of the table with the same pages to the last: a group whose members have everything but their last tokens' page in common, and share that too."""
    b = Batch([(64, [(5, 1), (5, 1)])], 8, 2, 64, 16, BF)
    b.table[1] = b.table[0]
    b.q[1] = b.q[0]
    b.check()
    assert b.way(GROUPS) == 0 and torch.equal(b.out[0], b.out[1])

"""What the operators for requests that share prefixes have to keep at their limits: of waits, of the scratch, of 32 bits, of pages (needs a B200).

Tolerances: `paged_reference.attention` derives its own.
"""
import random

import pytest
import torch

from paper_2604_18396_b200 import binding, cache_ops, prefix_attention_bytes
from tests import paged_reference as ref
from tests.test_gpu_prefix_attention import ALL, BF, F16, NAN, WHOLE, Batch, i32
from tests.test_gpu_prefix_batches import run_admit, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F16])
def test_waits_last_while_rows_are_computed_again(dtype):
    """300 prompts of two tokens behind the same 4094 positions, two units of 256 rows to a CTA; the last value, which only the second token sees, is infinite.
    Each part with it takes some 60 ms, a hundred times as long as 4096 polls of the warps that wait for its end may be counted upon."""
    n, seqs = 4096, 300
    b = Batch([(0, [(n - 2, 2)])], 128, 1, 64, 64, dtype)
    page = b.table[0, n // 64 - 1].long()
    b.pool[0, page, 1, 0, 63, 3] = 0.0
    want, tol = ref.attention(b.q, b.starts, b.pool, 1, b.table, b.lens, ALL, 0, b.scale)
    b.pool[0, page, 1, 0, 63, 3] = float("inf")
    b.lens, b.starts = [n] * seqs, list(range(0, 2 * seqs + 1, 2))
    b.table, b.lens_t, b.q_start, b.lead, b.shared = b.table.repeat(seqs, 1), i32(b.lens), i32(b.starts), i32(list(range(seqs))), i32([0] * seqs)
    b.q = b.q.repeat(seqs, 1, 1)
    b.out = torch.full_like(b.q, NAN)
    assert b.way(WHOLE, polls=4096) == 0
    assert b.status.item() == 0
    out = b.out.double().view(seqs, 2, 128, 64)
    assert (out[:, 1, :, 3] == float("inf")).all()
    out[:, 1, :, 3] = want[1, :, 3]
    assert ((out - want).abs() <= tol).all()


@pytest.mark.parametrize("big", [2048.0, 8192.0, 32768.0])
def test_equal_scores_of_many_millions_on_both_sides(big):
    """One key of the shared positions and one of each sequence's own score the same 2^25 and more, all others far less: the mean of their two values.

    Queries and keys are powers of two, so every way has the same score to the last bit, and the probabilities are 1/2 and 1/2 (exact in every type): what is
    left is one rounding of the result and a few of 32 bits."""
    for dtype in (F16, BF):
        b = Batch([(160, [(4, 1), (30, 1), (300, 1)])], 4, 2, 64, 16, dtype)
        b.q.fill_(big)
        b.pool[0, :, 0] = torch.where(torch.isnan(b.pool[0, :, 0]), b.pool[0, :, 0], 1.0)
        b.pool[0, b.table[0, 3].long(), 0, :, 7] = big  # position 55, for all
        for s, at in enumerate((161, 175, 400)):
            b.pool[0, b.table[s, at // 16].long(), 0, :, at % 16] = big
        for way in b.ways():
            b.out.fill_(NAN)
            assert b.way(way) == 0 and b.status.item() == 0
            for s, at in enumerate((161, 175, 400)):
                v = torch.stack((b.pool[0, b.table[0, 3].long(), 1, :, 7], b.pool[0, b.table[s, at // 16].long(), 1, :, at % 16])).double()
                want = v.mean(0).repeat_interleave(2, 0)
                bound = torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -20 * v.abs().sum(0).repeat_interleave(2, 0)
                assert ((b.out[s].double() - want).abs() <= bound).all(), (dtype, way, s)


def test_one_workspace_for_large_and_small_calls():
    """Sized for the largest batch, taken for all: prompts, a few tokens each, single tokens."""
    most = prefix_attention_bytes(16, 1200, 16, 4, 128)
    work = torch.full((most,), 0xff, dtype=torch.uint8, device="cuda")
    for members in ([(0, 75)] * 16, [(10 * i, 40) for i in range(16)], [(i, 60) for i in range(12)], [(3 * i, 9) for i in range(16)], [(5 * i, 1) for i in range(16)]):
        b = Batch([(512, members)], 16, 4, 128, 16, BF)
        b.table = torch.nn.functional.pad(b.table, (0, 2048 - b.table.shape[1]), value=-1)
        want, tol = b.statement()
        for own in (1, 100, 0):
            b.out.fill_(NAN)
            b.call(workspace=work, max_own=own)
            assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all(), (len(members), own)


@pytest.mark.parametrize("members", [[(5 * i, 1) for i in range(60)], [(i, 9) for i in range(16)], [(7 * i, 90) for i in range(5)], [(300, 700)]])
def test_nothing_is_written_behind_what_a_call_needs(members):
    b = Batch([(512, members)], 16, 4, 128, 16, BF)
    want, tol = b.statement()
    for width in (b.table.shape[1], 2048):
        b.table = torch.nn.functional.pad(b.table, (0, width - b.table.shape[1]), value=-1)
        for own in (1, 400, 0):
            c = cache_ops._cache(b.pool, b.table, b.lens_t, 0)
            n = binding.load().river_prefix_attention_needs(c, b.q.shape[0], b.max_q, own, 16)
            work = torch.full((n + (1 << 20),), 0x5a, dtype=torch.uint8, device="cuda")
            b.out.fill_(NAN)
            b.call(workspace=work[:n], max_own=own)
            assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all(), (width, own)
            assert (work[n:] == 0x5a).all(), (width, own)
            b.out.fill_(NAN)
            b.call(max_own=own)
            assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all(), (width, own)


@pytest.mark.parametrize("dtype", [BF, F16])
def test_rows_behind_max_q_hold_their_result_or_what_they_held(dtype):
    """By the way with single tokens nobody computes them, and the scratch (NaN) is not theirs."""
    b = Batch([(64, [(4, 1), (20, 4), (0, 3)]), (32, [(9, 2), (7, 3)])], 8, 2, 64, 16, dtype)
    want, tol = b.statement()
    b.max_q = 2
    for way in b.ways():
        b.out.fill_(7.0)
        b.status.zero_()
        assert b.way(way) == 0 and b.status.item() == -1
        right = ((b.out.double() - want).abs() <= tol).all(-1).all(-1)
        stayed = (b.out == 7.0).all(-1).all(-1)
        behind = torch.zeros_like(right)
        for s, n in enumerate((1, 4, 3, 2, 3)):
            behind[b.starts[s] + 2:b.starts[s] + n] = True
        assert (right | (stayed & behind)).all(), way


def test_admission_refused_leaves_the_state():
    """Too few pages; one row too short, by a position and by all that 32 bits hold: each by itself, in a table that the deciding CTA writes alone."""
    rng = random.Random(4)
    table, lens, refs = state(rng, 5, 10, 16, 60, share=0)
    refs = [max(r, int(i >= 20)) for i, r in enumerate(refs)]
    free = sum(r == 0 for r in refs)
    # (nobody begins with anything: what was held is free again, but for ids from 20 on that nobody held)
    given_back = sum(-(-n // 16) for n in lens)
    assert 5 * 10 > free + given_back
    for total in ([160] * 5, [0, 0, 161, 0, 0], [16, 0, 0, 0, 161], [2 ** 31 - 1] * 5, [0, 2 ** 31 - 1, 0, 0, 0]):
        assert run_admit(table, lens, refs, [-1] * 5, [0] * 5, total, 16) == [table, lens, refs, [0] * 5, -4], total

"""Attention over shared prefixes against the plain 64-bit statement, by each of its ways (needs a B200).

Tolerances: `paged_reference.attention` derives its own: one rounding of the result, one of every probability, and the fp32 arithmetic.  Parts of a row
that are joined add one fp32 rounding per part to the sums, which the term for the sums' length covers.
"""
import ctypes as C

import pytest
import torch

from paper_2604_18396_b200 import binding, cache_ops, prefix_attention, prefix_attention_bytes
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16
NAN = float("nan")
ALL = 1 << 29  # a window over everything
STEP, GROUPS, BOTH, WHOLE = range(4)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Batch:
    """groups: [(shared positions, [(positions of its own before the new ones, new ones)])]; pool filled with NaN where nobody has a position."""

    def __init__(self, groups, hq, hkv, dh, page, dtype, *, seed=3, layers=1, layer=1, size=2.0):
        self.lens, self.starts, lead, shared = [], [0], [], []
        for sh, members in groups:
            first = len(self.lens)
            for own, n in members:
                self.lens.append(sh + own + n)
                self.starts.append(self.starts[-1] + n)
                lead.append(first if len(members) > 1 or sh else len(self.lens) - 1)
                shared.append(sh)
        self.pool, self.table, self.lens_t = ref.cache(self.lens, page, hkv, dh, dtype, seed, layers=layers, layer=layer)
        for s, (l, sh) in enumerate(zip(lead, shared)):
            self.table[s, : sh // page] = self.table[l, : sh // page]
        self.lead, self.shared, self.q_start, self.layer = i32(lead), i32(shared), i32(self.starts), layer
        g = torch.Generator().manual_seed(seed + 1)
        self.q = (torch.randn(self.starts[-1], hq, dh, generator=g) * size).to(dtype).cuda()
        self.out, self.status = torch.full_like(self.q, NAN), i32([0])
        self.max_q, self.scale = max(n for _, m in groups for _, n in m), dh ** -0.5

    def call(self, **kw):
        kw = {"max_q": self.max_q, "status": self.status, "softmax_scale": self.scale, **kw}
        prefix_attention(self.q, self.out, self.q_start, self.pool, self.layer, self.table, self.lens_t, self.lead, self.shared, **kw)
        return self.out

    def way(self, way, mute=-1, polls=1 << 20):
        """The same call by one way; the return code."""
        t, hq, dh = self.q.shape
        c = cache_ops._cache(self.pool, self.table, self.lens_t, 0)
        self.work = torch.empty(prefix_attention_bytes(len(self.lens), t, hq, self.pool.shape[3], dh), dtype=torch.uint8, device="cuda")
        self.work.fill_(0xff)  # (NaN and -1: what the scratch holds before does not matter)
        return binding.load().river_selftest_prefix_attention(
            c, self.layer, t, self.max_q, self.q_start.data_ptr(), self.lead.data_ptr(), self.shared.data_ptr(), hq, cache_ops._rows(self.q, 0, "q"),
            C.c_float(self.scale), self.out.data_ptr(), self.work.data_ptr(), self.work.nbytes, self.status.data_ptr(), way, mute, polls,
            torch.cuda.current_stream().cuda_stream)

    def statement(self):
        return ref.attention(self.q, self.starts, self.pool, self.layer, self.table, self.lens, ALL, 0, self.scale)

    def ways(self):
        span = 2 * (128 // (self.q.shape[1] // self.pool.shape[3]))
        return [STEP, GROUPS, BOTH, WHOLE] if self.q.shape[0] < len(self.lens) * span else [STEP, WHOLE]

    def check(self, ways=None, status=0):
        want, tol = self.statement()
        for way in ways if ways is not None else self.ways():
            self.out.fill_(NAN)
            self.status.zero_()
            assert self.way(way) == 0
            assert self.status.item() == status, way
            far = (self.out.double() - want).abs() - tol
            assert (far <= 0).all(), (way, far.max().item(), (~(far <= 0)).nonzero()[:5].tolist())
        self.out.fill_(NAN)
        self.status.zero_()
        self.call()
        assert self.status.item() == status and ((self.out.double() - want).abs() <= tol).all()


CASES = {
    "one_token": ([(0, [(0, 1)])], 8, 2, 64, 16, BF),
    "two_tokens_one_page": ([(16, [(0, 1), (0, 1)])], 4, 2, 64, 16, F16),
    "four_beams": ([(160, [(3, 1), (4, 1), (15, 1), (16, 1)])], 32, 8, 64, 16, BF),
    "one_kv_head": ([(320, [(40, 1)] * 6)], 12, 1, 128, 32, F16),
    "as_many_kv_heads": ([(640, [(7, 1), (70, 1), (700, 1)])], 4, 4, 128, 64, BF),
    "dual_and_more_rows": ([(1008, [(i, 1) for i in range(40)])], 16, 4, 128, 16, BF),
    "seven_heads_to_one": ([(2000, [(11 * i, 1) for i in range(25)])], 14, 2, 64, 16, F16),
    "groups_and_loners": ([(0, [(300, 1)]), (512, [(1, 1), (90, 1), (33, 1)]), (0, [(0, 1)]), (48, [(0, 1), (500, 1)]), (0, [(77, 1)])], 8, 2, 128, 16, BF),
    "alone_with_a_prefix": ([(256, [(5, 1)]), (64, [(9, 1), (9, 1)])], 8, 2, 64, 16, BF),
    "without_new_tokens": ([(128, [(8, 0), (5, 1), (9, 0)]), (64, [(3, 0), (2, 0)]), (0, [(50, 1), ]), (32, [(1, 0), (1, 2)])], 8, 4, 64, 16, F16),
    "few_tokens_each": ([(400, [(0, 3), (20, 5), (1, 1), (300, 9)]), (96, [(0, 2), (0, 2)])], 16, 4, 128, 16, BF),
    "prompts": ([(304, [(0, 60), (100, 33), (7, 129)]), (0, [(0, 200)])], 16, 4, 128, 16, BF),
    "prompts_of_many_heads": ([(128, [(3, 20), (0, 41)]), (64, [(0, 5), (60, 90)])], 60, 1, 64, 32, F16),
    "a_hundred_and_twentyeight_heads": ([(256, [(0, 1), (9, 1), (30, 3)])], 128, 1, 64, 16, BF),
    "long_prompts": ([(1024, [(0, 700), (513, 300)])], 8, 2, 128, 64, F16),
    "many_sequences": ([(16 * (g % 4), [(g % 7, 1)] * (1 + g % 3)) for g in range(260)], 4, 1, 64, 16, BF),
    "page_of_64": ([(64 * 9, [(i, 1) for i in range(0, 130, 10)])], 24, 8, 128, 64, F16),
}


@pytest.mark.parametrize("name", CASES)
def test_results_by_every_way(name):
    Batch(*CASES[name]).check()


def test_longer_than_every_cta_once():
    """A prefix that all CTAs share out, rows of two query tiles, and sequences that split over a cluster."""
    Batch([(9008, [(37 * i, 1) for i in range(48)])], 16, 2, 128, 16, BF).check()


def test_block_of_a_pool_of_several_and_strided_queries():
    b = Batch([(208, [(9, 1), (30, 2), (2, 1)])], 8, 2, 64, 16, BF, layers=3, layer=2)
    x = torch.randn(b.q.shape[0], 3, 8, 80, device="cuda").to(BF)
    b.q = x[:, 1, :, 8:72]  # heads 80 apart, tokens 1920
    b.check()
    b.q = x[:, 0, :, :64].transpose(0, 1).contiguous().transpose(0, 1)  # heads before tokens
    b.check()


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    for dtype in (BF, F16):
        b = Batch([(176, [(0, 1), (20, 3), (40, 1)])], 8, 2, 64, 16, dtype)
        b.scale = scale
        b.check()


@pytest.mark.parametrize("dtype", [BF, F16])
def test_rising_scores(dtype):
    """Every key larger than those before it: the maximum moves in every tile, up to scores of many thousands."""
    b = Batch([(1600, [(50, 1), (200, 2), (3, 1)])], 4, 2, 64, 16, dtype)
    b.q.fill_(1.0)
    for s in range(3):
        for j in range(b.lens[s]):
            b.pool[0, b.table[s, j // 16], 0, :, j % 16] = j / 16.0
    b.check()


@pytest.mark.parametrize("dtype", [BF, F16])
def test_values_that_are_infinite(dtype):
    """An infinite value that is seen gives infinity, one that is hidden or of another sequence nothing."""
    b = Batch([(160, [(4, 1), (9, 3), (40, 1)])], 8, 2, 64, 16, dtype)
    page = b.table[0, 2].long()
    b.pool[0, page, 1, 0, 5, 3] = float("inf")           # shared: everybody's
    b.pool[0, b.table[1, 10].long(), 1, 1, 11, 7] = float("-inf")  # position 171 of the second sequence: only its last token's
    want, _ = b.statement()
    hidden = b.pool[0, b.table[1, 10].long(), 1, 1, 11, 7].clone()
    b.pool[0, b.table[1, 10].long(), 1, 1, 11, 7] = 0.0  # (the statement multiplies hidden values by 0: for the rows that do not see this one)
    without, _ = b.statement()
    b.pool[0, b.table[1, 10].long(), 1, 1, 11, 7] = hidden
    want[:3] = without[:3]
    for way in b.ways():
        b.out.fill_(NAN)
        assert b.way(way) == 0 and b.status.item() == 0
        assert torch.equal(torch.isinf(b.out), torch.isinf(want)) and not torch.isnan(b.out).any(), way
        ok = ~torch.isinf(want)
        assert (b.out.double() - want)[ok].abs().max() < 0.1, way
        assert (b.out[:, :4, 3] == float("inf")).all() and (b.out[3, 4:, 7] == float("-inf")).all() and torch.isfinite(b.out[:3, 4:]).all()


def test_keys_that_are_no_numbers():
    """A key that is no number makes the rows that see it no numbers, and no others."""
    b = Batch([(64, [(4, 1), (9, 3)]), (64, [(0, 1), (1, 1)])], 4, 2, 64, 16, BF)
    b.pool[0, b.table[0, 1].long(), 0, 1, 5, 3] = NAN          # the first group's, KV head 1
    b.pool[0, b.table[1, 4].long(), 0, 0, 11, 3] = NAN         # position 75, the last one of the second sequence, KV head 0
    for way in b.ways():
        b.out.fill_(0)
        assert b.way(way) == 0
        bad = torch.isnan(b.out).all(-1)
        assert torch.equal(bad, torch.isnan(b.out).any(-1))
        want = torch.zeros_like(bad)
        want[:4, 2:] = True
        want[3, :2] = True
        assert torch.equal(bad, want), way


@pytest.mark.parametrize("dtype,big", [(BF, 2.0e4), (F16, 3.0e3)])
def test_scores_of_many_millions(dtype, big):
    """Where rounding a maximum weighs more than an exponent has room for, rows are computed one by one: the largest score takes everything."""
    b = Batch([(160, [(4, 1), (30, 2), (0, 1)])], 4, 2, 64, 16, dtype)
    b.q.fill_(big)
    b.pool[0, :, 0] = torch.where(torch.isnan(b.pool[0, :, 0]), b.pool[0, :, 0], 1.0)
    b.pool[0, b.table[0, 3].long(), 0, :, 7] = big  # position 55, for all
    row = b.pool[0, b.table[0, 3].long(), 1, :, 7].repeat_interleave(2, 0)
    for way in b.ways():
        b.out.fill_(NAN)
        assert b.way(way) == 0 and torch.equal(b.out, row.expand_as(b.out)), way


def test_missing_pages_count_as_not_visible():
    b = Batch([(160, [(4, 1), (40, 3), (0, 1)])], 8, 2, 64, 16, BF)
    keep = b.table.clone()
    for s, col, bad in ((0, 3, -1), (1, 11, 1 << 30)):  # of the group, of a sequence
        b.table.copy_(keep)
        b.table[s, col] = bad
        at = list(range(3 * 16, 4 * 16)) if s == 0 else list(range(176, 192))
        for way in b.ways():
            b.out.fill_(NAN)
            b.status.zero_()
            assert b.way(way) == 0 and b.status.item() == -1
            for i in range(3):
                for t in range(b.starts[i], b.starts[i + 1]):
                    p = b.lens[i] - (b.starts[i + 1] - t)
                    # by the first way the other sequences read their own row of the table, where the page stands
                    hidden = at if i == s or (s == 0 and way in (GROUPS, BOTH)) else []
                    j = torch.tensor([x for x in range(p + 1) if x not in hidden], device="cuda")
                    kv = b.pool[0, keep[i].long()[j // 16], :, :, j % 16].double()
                    for h in range(8):
                        w = torch.softmax(kv[:, 0, h // 4] @ b.q[t, h].double() * b.scale, 0)
                        x = w @ kv[:, 1, h // 4]
                        assert ((b.out[t, h].double() - x).abs() <= 2.0 ** -8 * (x.abs() + w @ kv[:, 1, h // 4].abs()) * 1.01 + 1e-5).all(), (way, i, t, h)


def test_queries_before_position_zero():
    """More queries than positions: those before position 0 see nothing."""
    b = Batch([(0, [(0, 5)]), (0, [(0, 3)])], 4, 2, 64, 16, BF)
    b.lens = [3, 0]
    b.lens_t = i32(b.lens)
    b.check(ways=[STEP, GROUPS, BOTH, WHOLE])


def test_arrays_that_are_not_as_described():
    """Told, and nothing outside the rows written: descending starts, lengths out of range, groups that are none."""
    def fresh():
        return Batch([(64, [(4, 1), (20, 1), (0, 1)]), (0, [(9, 1)])], 4, 2, 64, 16, BF)

    for change in (lambda b: b.q_start.copy_(i32([0, 2, 1, 3, 4])), lambda b: b.lens_t.copy_(i32([-5, 85, 65, 10])), lambda b: b.lens_t.copy_(i32([1 << 20, 85, 65, 10])),
                   lambda b: b.lead.copy_(i32([0, 0, 1, 3])), lambda b: b.lead.copy_(i32([0, 0, -7, 3])), lambda b: b.lead.copy_(i32([0, 0, 1 << 30, 3])),
                   lambda b: b.lead.copy_(i32([2, 2, 2, 3])), lambda b: b.shared.copy_(i32([64, 48, 64, 0])), lambda b: b.shared.copy_(i32([65, 65, 65, 0])),
                   lambda b: b.shared.copy_(i32([-64, -64, -64, 0])), lambda b: b.shared.copy_(i32([80, 80, 80, 0])), lambda b: b.lens_t.copy_(i32([69, 85, 64, 10]))):
        for way in (GROUPS, BOTH):
            b = fresh()
            change(b)
            whole = torch.zeros(6, 4, 64, dtype=BF, device="cuda")
            b.out = whole[1:5]
            assert b.way(way) == 0
            torch.cuda.synchronize()
            assert b.status.item() == -1 and (whole[0] == 0).all() and (whole[5] == 0).all()


def test_more_queries_than_max_q():
    b = Batch([(64, [(4, 1), (20, 3)])], 4, 2, 64, 16, BF)
    want, tol = b.statement()
    b.max_q = 2
    for way in b.ways():
        b.out.fill_(NAN)
        b.status.zero_()
        assert b.way(way) == 0 and b.status.item() == -1
        assert ((b.out.double() - want).abs() <= tol)[:3].all()


def test_the_same_bits_twice():
    b = Batch([(4000, [(50 * i, 1) for i in range(30)]), (640, [(3, 2)] * 9)], 8, 2, 128, 16, BF)
    for way in b.ways():
        assert b.way(way) == 0
        first = b.out.clone()
        assert b.way(way) == 0 and torch.equal(first, b.out)


def test_a_wait_that_runs_out_is_told():
    b = Batch([(640, [(4, 1), (20, 1)])], 8, 2, 64, 16, BF)
    for way in (GROUPS, BOTH, WHOLE):
        b.status.zero_()
        assert b.way(way, mute=0, polls=64) == 0
        assert b.status.item() == -7
        b.status.zero_()
        assert b.way(way) == 0 and b.status.item() == 0
    b.check()


def test_other_streams_graphs_and_two_calls_at_once():
    b, c = (Batch([(1200, [(10 * i, 1) for i in range(9)])], 8, 2, 128, 16, BF, seed=s) for s in (5, 6))
    wb, wc = b.statement(), c.statement()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        b.call(stream=s1)
        c.call(stream=s2)
    torch.cuda.synchronize()
    for x, (want, tol) in ((b, wb), (c, wc)):
        assert x.status.item() == 0 and ((x.out.double() - want).abs() <= tol).all()
    work = torch.empty(prefix_attention_bytes(9, 9, 8, 2, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # two calls, one after the other, on one workspace
        b.call(workspace=work)
        c.call(workspace=work)
    for seed in (1, 2):
        b.out.fill_(NAN)
        c.out.fill_(NAN)
        b.q.copy_(torch.randn(b.q.shape, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        for x in (b, c):
            want, tol = x.statement()
            assert ((x.out.double() - want).abs() <= tol).all()


def test_rows_behind_the_last_sequence_stay():
    """A batch padded to a fixed number of rows, as a captured step has it."""
    b = Batch([(320, [(4, 1), (20, 1), (9, 2)]), (0, [(70, 1)])], 8, 2, 64, 16, BF)
    want, tol = b.statement()
    t = b.q.shape[0]
    b.q, b.out = torch.cat((b.q, torch.full((40, 8, 64), NAN, dtype=BF, device="cuda"))), torch.empty(t + 40, 8, 64, dtype=BF, device="cuda")
    for way in [None] + b.ways():
        b.out.fill_(7.0)
        if way is None:
            b.call()
        else:
            assert b.way(way) == 0
        assert b.status.item() == 0 and ((b.out[:t].double() - want).abs() <= tol).all() and (b.out[t:] == 7.0).all(), way


def test_one_long_prompt_among_many_single_tokens():
    """Places of queries that are none, by the million: not a grid of single tokens."""
    b = Batch([(64, [(3, 1)] * 200 + [(0, 900)] + [(5, 1)] * 100)], 4, 2, 64, 16, BF)
    want, tol = b.statement()
    b.call()
    assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all()
    b.out.fill_(NAN)
    b.call(max_q=2 ** 31 - 1)  # (as many as there are rows)
    assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("max_own", [0, 1, 100, 5000, 2 ** 31 - 1])
def test_whatever_the_caller_expects(max_own):
    for groups in ([(2000, [(30 * i, 1) for i in range(20)])], [(48, [(9, 30), (0, 2)])]):
        b = Batch(groups, 8, 2, 128, 16, F16)
        want, tol = b.statement()
        b.call(max_own=max_own)
        assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all()


def test_a_workspace_of_the_callers():
    b = Batch([(1008, [(5 * i, 1) for i in range(64)])], 8, 2, 128, 16, BF)
    b.table = torch.nn.functional.pad(b.table, (0, 4096 - b.table.shape[1]), value=-1)  # (by the table's width, groups pay)
    want, tol = b.statement()
    n = prefix_attention_bytes(64, 64, 8, 2, 128)
    work = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    b.call(workspace=work, max_own=400)
    assert b.status.item() == 0 and ((b.out.double() - want).abs() <= tol).all()
    with pytest.raises(binding.RiverError):
        b.call(workspace=work[: n - 128], max_own=400)
    for bad in (work.view(torch.int32), work.view(2, -1)[:, :5], work.cpu()):
        with pytest.raises(ValueError):
            b.call(workspace=bad)


def test_no_tokens():
    b = Batch([(64, [(4, 1), (20, 1)])], 4, 2, 64, 16, BF)
    b.q, b.out = b.q[:0], b.out[:0]
    b.q_start.zero_()
    b.call(max_q=1)
    torch.cuda.synchronize()

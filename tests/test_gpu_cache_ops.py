"""The operators on a caller's paged cache against plain 64-bit statements: rotary positions written into pages, windowed attention with
sinks, pages that grow, slide, fork and move (needs a B200).

Tolerances: `paged_reference.attention` derives its own; a turned value is one rounding of the result plus fp32 arithmetic on values
whose sine and cosine are off by at most 2^-22; pages' bookkeeping and moved values are exact.
"""
import random

import pytest
import torch

from paper_2604_18396_b200 import pages_advance, pages_compact, pages_reorder, rope_append, window_attention
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN = float("nan")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- rotary positions
@pytest.mark.parametrize("t,hq,hkv,dh,rot,inter,tin,tc,page,packed", [
    (1, 32, 8, 128, 128, False, BF, BF, 16, True), (1, 1, 1, 64, 2, True, F32, F16, 64, True), (7, 6, 2, 64, 64, True, BF, BF, 16, False),
    (33, 24, 8, 128, 96, False, F32, BF, 32, True), (5, 3, 1, 128, 34, False, F16, F16, 16, False), (64, 8, 8, 64, 48, True, F16, F16, 64, True),
    (130, 4, 4, 128, 18, True, F32, F16, 16, False), (19, 16, 2, 128, 128, True, F32, BF, 16, True), (300, 7, 1, 64, 62, False, BF, BF, 32, True)])
def test_rope_append(t, hq, hkv, dh, rot, inter, tin, tc, page, packed):
    g = torch.Generator().manual_seed(t + dh + rot)
    seqs_n = min(t, 5)
    lens = [3 + 97 * s for s in range(seqs_n)]
    counts = [len(range(s, t, seqs_n)) for s in range(seqs_n)]
    pool, table, _ = ref.cache([n + c for n, c in zip(lens, counts)], page, hkv, dh, tc, 5, layers=2, layer=1)
    seqs = torch.arange(t) % seqs_n
    positions = torch.tensor([lens[t_ % seqs_n] + t_ // seqs_n for t_ in range(t)])
    if packed:
        x = torch.randn(t, (hq + 2 * hkv) * dh, generator=g).to(tin).cuda()
        q, k, v = (y.unflatten(-1, (-1, dh)) for y in x.split([hq * dh, hkv * dh, hkv * dh], -1))
    else:  # heads before tokens, in memory that starts off every 16-byte boundary
        x = torch.randn(1 + (hq + 2 * hkv) * t * dh, generator=g).to(tin).cuda()[1:].view(hq + 2 * hkv, t, dh).transpose(0, 1)
        q, k, v = x.split([hq, hkv, hkv], 1)
    f = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()
    want_pool = pool.clone()
    q_out, status = torch.full((t, hq, dh), NAN, dtype=tc, device="cuda"), i32([0])
    rope_append(q, k, v, positions.int().cuda(), seqs.int().cuda(), f, pool, 2, table, q_out, interleaved=inter, scale=1.25, status=status)
    assert status.item() == 0
    u, pos = ref.U[tc], positions.cuda()

    def near(got, x):
        want = ref.rope(x, pos, f, inter, 1.25)
        # (the pair's length bounds what an error of sine and cosine, and the two products' roundings, amount to)
        size = 1.25 * (x.double().abs().amax(-1, keepdim=True) * 2)
        assert ((got.double() - want).abs() <= u * want.abs() + 2.0 ** -21 * size + ref.TINY[tc]).all()
        assert torch.equal(got[..., rot:], x[..., rot:].to(tc))

    near(q_out, q)
    page_of = table.long()[seqs.cuda(), pos // page]
    near(pool[1, page_of, 0, :, pos % page], k)
    assert torch.equal(pool[1, page_of, 1, :, pos % page], v.to(tc))
    # nothing else has changed
    want_pool[1, page_of, :, :, pos % page] = pool[1, page_of, :, :, pos % page]
    assert torch.equal(pool.view(torch.int16), want_pool.view(torch.int16))


def test_rope_append_far_positions_keep_their_angles():
    """An angle of 10^8 radians, to fp32."""
    t, dh = 64, 128
    pool = torch.zeros(1, 1, 2, 1, 16, dh, dtype=F16, device="cuda")
    q = torch.randn(t, 4, dh, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    pos = torch.randint(90_000_000, 100_000_000, (t,), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    f = (10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64) / dh)).float().cuda()
    q_out = torch.empty(t, 4, dh, dtype=F16, device="cuda")
    kv = torch.zeros(t, 1, dh, device="cuda")
    status = i32([0])
    rope_append(q, kv, kv, pos, i32([0] * t), f, pool, 1, i32([[0]]), q_out, status=status)
    assert status.item() == -1  # (no such pages: queries turn all the same)
    want = ref.rope(q, pos, f, False, 1.0)
    assert ((q_out.double() - want).abs() <= ref.U[F16] * want.abs() + 2.0 ** -21 * 2 * q.abs().max()).all()
    assert (pool == 0).all()


def test_rope_append_padding_and_tokens_without_a_place():
    pool, table, _ = ref.cache([40, 20], 16, 2, 64, BF, 3, fill=0.0)
    before = pool.clone()
    table[1, 1] = -1
    k = torch.randn(6, 2, 64, device="cuda", dtype=BF)
    q = torch.randn(6, 4, 64, device="cuda", dtype=BF)
    f = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda()
    #         fine, padding, page -1, sequence 2 of 2, position -3, behind the table
    seqs, pos = i32([0, -1, 1, 2, 0, 0]), i32([5, 7, 17, 0, -3, 16 * table.shape[1]])
    q_out = torch.full_like(q, NAN)
    status = i32([0])
    rope_append(q[:2], k[:2], k[:2], pos[:2], seqs[:2], f, pool, 1, table, q_out[:2], status=status)
    assert status.item() == 0 and (q_out[1] == 0).all()
    assert torch.equal(pool[0, table[0, 0].long(), 1, :, 5], k[0])
    pool.copy_(before)
    for i in range(2, 6):
        status.zero_()
        rope_append(q[i:i + 1], k[i:i + 1], k[i:i + 1], pos[i:i + 1], seqs[i:i + 1], f, pool, 1, table, q_out[i:i + 1], status=status)
        assert status.item() == -1 and torch.equal(pool, before), i
        want = ref.rope(q[i:i + 1], pos[i:i + 1], f, False, 1.0)
        assert ((q_out[i:i + 1].double() - want).abs() <= ref.U[BF] * want.abs() + 2.0 ** -19 * q[i].abs().max()).all()
    # no queries: keys and values alone
    rope_append(None, k, k, i32([0, 1, 2, 3, 4, 5]), i32([0] * 6), f, pool, 1, table, None)
    assert torch.equal(pool[0, table[0, 0].long(), 1, :, :6].transpose(0, 1), k)


# ---------------------------------------------------------------- attention
def attn_case(new, hist, hq, hkv, dh, page, window, sinks, dtype, *, seed=0, layers=2, layer=2, hide=NAN, head_major=False, scale=None, drop=True):
    """Runs the operator with everything that no query sees set to `hide` and its pages dropped, and compares with the reference."""
    lens = [a + b for a, b in zip(new, hist)]
    pool, table, lens_t = ref.cache(lens, page, hkv, dh, dtype, seed, layers=layers, layer=layer, fill=hide)
    g = torch.Generator().manual_seed(seed + 1)
    t = sum(new)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    q = (torch.randn(hq, t, dh, generator=g) * 2).to(dtype).cuda().transpose(0, 1) if head_major else (
        torch.randn(t, hq + 3, dh, generator=g) * 2).to(dtype).cuda()[:, :hq]
    scale = dh ** -0.5 if scale is None else scale
    want, tol = ref.attention(q, starts, pool, layer, table, lens, window, sinks, scale)
    for s, n in enumerate(lens):
        if n == 0:
            continue
        seen = ref.visible(n, new[s], window, sinks, "cpu").any(0) if new[s] else torch.zeros(n, dtype=torch.bool)
        for j in range(-(-n // page)):
            m = seen[j * page:(j + 1) * page]
            p = int(table[s, j])
            if drop and not m.any():
                table[s, j] = -1
            pool[layer - 1, p, :, :, : len(m)][:, :, ~m.cuda()] = hide
    out, status = torch.full((t, hq, dh), NAN, dtype=dtype, device="cuda"), i32([0])
    window_attention(q, out, i32(starts), pool, layer, table, lens_t, window=window, sinks=sinks, max_q=max(new), softmax_scale=scale, status=status)
    assert status.item() == 0
    assert out.isfinite().all()
    over = (out.double() - want).abs() - tol
    assert (over <= 0).all(), (over.max().item(), (over > 0).sum().item())
    again = torch.empty_like(out)
    window_attention(q, again, i32(starts), pool, layer, table, lens_t, window=window, sinks=sinks, max_q=max(new) + 3, softmax_scale=scale)
    return out, again


STEP = [
    # lengths of 0, 1 and around pages and windows; a sequence without a query
    ([1, 1, 1, 1, 0, 1, 1], [0, 1, 15, 16, 9, 63, 200], 4, 1, 128, 16, 32, 4, BF),
    ([1] * 9, [0, 6, 7, 8, 9, 31, 32, 33, 500], 8, 8, 64, 16, 8, 0, F16),
    ([1] * 5, [3, 30, 64, 700, 1030], 24, 8, 128, 32, 200, 20, F16),
    ([1] * 3, [0, 100, 1500], 32, 8, 64, 64, 1024, 4, BF),
    ([1] * 4, [5, 18, 40, 333], 7, 1, 128, 16, 1, 0, BF),
    ([1] * 4, [5, 18, 40, 333], 7, 1, 64, 16, 1, 33, BF),
    ([1] * 2, [2000, 2500], 12, 1, 128, 64, 100000, 0, BF),
    ([1] * 2, [2000, 2500], 16, 1, 64, 16, 513, 700, F16),
    ([1] * 40, list(range(40, 80)), 4, 2, 64, 16, 17, 1, BF),
    ([2, 3, 1], [100, 0, 60], 8, 2, 128, 16, 50, 3, BF),
]
PROMPT = [
    ([17, 0, 333, 40, 128], [0, 7, 50, 1111, 64], 24, 8, 128, 32, 200, 20, F16),
    ([64], [0], 4, 1, 128, 16, 1000, 0, BF),
    ([300], [0], 8, 8, 64, 16, 128, 4, BF),
    ([129, 255], [31, 0], 4, 4, 128, 16, 1, 0, BF),
    ([70, 90], [500, 3], 6, 2, 64, 64, 33, 65, F16),
    ([520], [777], 7, 1, 128, 16, 300, 130, BF),
    ([31, 100], [9, 260], 12, 1, 64, 16, 64, 16, BF),
    ([1500], [0], 2, 1, 128, 32, 700, 1, F16),
    ([600], [1000], 16, 4, 128, 16, 5000, 0, BF),
    ([200, 1, 2, 64], [0, 300, 4, 64], 32, 2, 64, 32, 48, 8, F16),
]


@pytest.mark.parametrize("new,hist,hq,hkv,dh,page,window,sinks,dtype", STEP + PROMPT)
def test_window_attention(new, hist, hq, hkv, dh, page, window, sinks, dtype):
    out, again = attn_case(new, hist, hq, hkv, dh, page, window, sinks, dtype)
    assert (out.double() - again.double()).abs().max() < 0.05  # (a larger max_q may take another kernel)


@pytest.mark.parametrize("hide", [float("inf"), -float("inf"), 65504.0])
@pytest.mark.parametrize("new,hist", [([1, 1, 1], [70, 9, 300]), ([90, 33], [70, 300])])
def test_window_attention_whatever_hidden_places_hold(new, hist, hide):
    attn_case(new, hist, 8, 2, 128, 16, 40, 5, F16, hide=hide, drop=False)
    attn_case(new, hist, 8, 2, 64, 32, 40, 5, BF, hide=hide, head_major=True)


def test_window_attention_same_bits_each_time():
    for new, hist in (([1] * 6, [900, 20, 4000, 333, 0, 77]), ([300, 77], [900, 20])):
        bits = set()
        for _ in range(4):
            out, _ = attn_case(new, hist, 8, 2, 128, 16, 512, 4, BF, seed=3)
            bits.add(out.view(torch.int16).cpu().numpy().tobytes())
        assert len(bits) == 1


@pytest.mark.parametrize("new,hist", [([1, 1], [200, 90]), ([3, 2], [200, 90]), ([100, 70], [200, 0])])
@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf")])
def test_window_attention_a_position_reaches_only_queries_that_see_it(new, hist, value):
    """One key or one value that is no number: queries that see it answer as the formula does, the others as if it were not there."""
    window, sinks, page, hq, hkv, dh = 30, 2, 16, 4, 2, 128
    lens = [a + b for a, b in zip(new, hist)]
    starts = [0, new[0], sum(new)]
    q = torch.randn(sum(new), hq, dh, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    for which in (0, 1):
        for s, j in ((0, lens[0] - 5), (0, lens[0] - new[0] - 10), (1, 1), (1, lens[1] - 1)):
            pool, table, lens_t = ref.cache(lens, page, hkv, dh, BF, 2, fill=0.0)
            clean, tol = ref.attention(q, starts, pool, 1, table, lens, window, sinks, dh ** -0.5)
            pool[0, table[s, j // page].long(), which, 1, j % page, 7] = value
            out = torch.empty_like(q)
            window_attention(q, out, i32(starts), pool, 1, table, lens_t, window=window, sinks=sinks, max_q=max(new))
            sees = torch.zeros(sum(new), dtype=torch.bool, device="cuda")
            sees[starts[s]:starts[s + 1]] = ref.visible(lens[s], new[s], window, sinks, "cuda")[:, j]
            far = (out.double() - clean).abs() <= tol
            assert far[~sees].all() and far[:, :2].all(), (which, s, j)
            hit = out[sees][:, 2:]
            if which == 1:  # a value: one dim of the result
                assert far[..., torch.arange(dh, device="cuda") != 7].all()
                assert (hit[..., 7].isnan() if value != value else hit[..., 7] == value).all()
            elif value != value:  # a key that is no number: no number anywhere
                assert hit.isnan().all()


def test_window_attention_missing_pages_count_as_hidden():
    pool, table, lens = ref.cache([100, 64], 16, 1, 64, BF, 4)
    q = torch.randn(2, 2, 64, device="cuda").to(BF)
    for bad in (-1, pool.shape[1], -7, 2 ** 31 - 1):
        t2 = table.clone()
        t2[0, 3] = bad
        t2[1, :] = bad  # a sequence that sees nothing
        out, status = torch.full_like(q, NAN), i32([0])
        window_attention(q, out, i32([0, 1, 2]), pool, 1, t2, lens, window=70, sinks=3, max_q=1, status=status)
        assert status.item() == -1 and (out[1] == 0).all()
        j = torch.tensor([j for j in range(100) if (j < 3 or j > 29) and j // 16 != 3], device="cuda")
        kv = pool[0, table[0].long()[j // 16], :, 0, j % 16].double()
        want = torch.softmax(q[0].double() @ kv[:, 0].T / 8, -1) @ kv[:, 1]
        assert ((out[0].double() - want).abs() < 0.02).all()
    # prompts
    q = torch.randn(80, 2, 64, device="cuda").to(BF)
    t2 = table.clone()
    t2[0, 3] = -1
    out, status = torch.full_like(q, NAN), i32([0])
    window_attention(q, out, i32([0, 80, 80]), pool, 1, t2, lens, window=70, sinks=3, max_q=80, status=status)
    assert status.item() == -1
    m = ref.visible(100, 80, 70, 3, "cuda")
    m[:, 48:64] = False
    k, v = (x.double() for x in ref.sequence(pool, 1, table, 0, 100))
    for h in range(2):
        sc = (q[:, h].double() @ k[:, 0].T / 8).masked_fill(~m, -float("inf"))
        assert ((out[:, h].double() - torch.softmax(sc, -1) @ v[:, 0]).abs() < 0.02).all()


def test_window_attention_more_queries_than_positions():
    """Queries before position 0 see nothing."""
    for new in (3, 60):
        pool, table, lens = ref.cache([2], 16, 1, 64, BF, 4)
        q = torch.randn(new, 4, 64, device="cuda").to(BF)
        out = torch.full_like(q, NAN)
        window_attention(q, out, i32([0, new]), pool, 1, table, lens, window=70, sinks=3, max_q=new)
        want, tol = ref.attention(q, [0, new], pool, 1, table, [2], 70, 3, 0.125)
        assert (out[: new - 2] == 0).all() and ((out.double() - want).abs() <= tol).all()


def test_window_attention_flags_a_wrong_max_q():
    pool, table, lens = ref.cache([50, 50], 16, 1, 64, BF, 4)
    for new, max_q in ((4, 1), (70, 40)):
        q = torch.zeros(new, 1, 64, device="cuda", dtype=BF)
        out, status = torch.zeros_like(q), i32([0])
        window_attention(q, out, i32([0, new, new]), pool, 1, table, lens, window=10, max_q=max_q, status=status)
        assert status.item() == -1
    out, status = torch.zeros_like(q), i32([0])
    window_attention(q, out, i32([0, 5, 3]), pool, 1, table, lens, window=10, max_q=5, status=status)
    assert status.item() == -1


def test_window_attention_lengths_beyond_the_table():
    pool, table, lens = ref.cache([64, 30], 16, 1, 64, BF, 4, width=4)
    q = torch.randn(60, 2, 64, device="cuda").to(BF)
    for new in (1, 60):
        want, got = torch.zeros_like(q), torch.full_like(q, NAN)
        window_attention(q, want, i32([0, new, new]), pool, 1, table, lens, window=20, sinks=2, max_q=new)
        status = i32([0])
        window_attention(q, got, i32([0, new, new]), pool, 1, table, i32([2 ** 31 - 1, 30]), window=20, sinks=2, max_q=new, status=status)
        assert status.item() == -1 and torch.equal(got[:new], want[:new])


@pytest.mark.parametrize("hq,hkv", [(160, 1), (129, 1), (128, 1)])
def test_window_attention_many_heads_to_one(hq, hkv):
    attn_case([20, 1], [100, 5], hq, hkv, 64, 16, 64, 4, BF)


def test_offsets_past_32_bits():
    """A block that begins 5 GB into the pool."""
    hkv, dh, page = 8, 128, 16
    n_pages = 40000
    pool = torch.zeros(3, n_pages, 2, hkv, page, dh, dtype=BF, device="cuda")  # 2.6 GB a block
    table = torch.arange(n_pages - 1, n_pages - 9, -1, dtype=torch.int32, device="cuda").view(1, 8)
    lens = i32([128])
    k, q = torch.randn(128, hkv, dh, device="cuda").to(BF), torch.randn(128, hkv, dh, device="cuda").to(BF)
    f = torch.zeros(64, device="cuda")
    q_out = torch.empty_like(q)
    rope_append(q, k, -k, torch.arange(128, dtype=torch.int32, device="cuda"), i32([0] * 128), f, pool, 3, table, q_out)
    assert torch.equal(q_out, q)
    got, _ = ref.sequence(pool, 3, table, 0, 128)
    assert torch.equal(got, k) and not pool[:2].any()
    for t0 in (0, 127):
        out = torch.empty_like(q[t0:])
        window_attention(q[t0:], out, i32([0, 128 - t0]), pool, 3, table, lens, window=50, sinks=2, max_q=128 - t0)
        want, tol = ref.attention(q[t0:], [0, 128 - t0], pool, 3, table, [128], 50, 2, dh ** -0.5)
        assert ((out.double() - want).abs() <= tol).all()
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[table[0].long()] = 1
    t2, r2, remap, n = torch.empty_like(table), torch.empty_like(refs), torch.empty_like(refs), i32([0])
    pages_compact(pool, table, refs, t2, r2, remap, n)
    assert n.item() == 8 and sorted(t2[0].tolist()) == list(range(8))
    got, neg = ref.sequence(pool, 3, t2, 0, 128)
    assert torch.equal(got, k) and torch.equal(neg, -k)


# ---------------------------------------------------------------- pages
def state(rng, seqs, width, page, n_pages, shared=True):
    """A random table whose sequences share some leading pages, its lengths and reference counts."""
    free = list(range(n_pages))
    rng.shuffle(free)
    table, lens, refs = [], [], [0] * n_pages
    for s in range(seqs):
        n = rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, width * page), rng.randint(0, width * page)])
        n = min(n, width * page, page * (len(free) // 2))
        row = [-1] * width
        lead = 0
        if shared and s and rng.random() < 0.5:
            o = rng.randrange(s)
            lead = rng.randint(0, min(n // page, lens[o] // page))
            row[:lead] = table[o][:lead]
        for j in range(lead, -(-n // page)):
            row[j] = free.pop()
        for j in range(-(-n // page)):
            if rng.random() < 0.03 and j < n // page:
                if j >= lead:
                    free.append(row[j])
                row[j] = -1
            elif row[j] >= 0:
                refs[row[j]] += 1
        table.append(row)
        lens.append(n)
    return table, lens, refs


@pytest.mark.parametrize("seqs,width,page,n_pages", [(1, 1, 16, 1), (1, 5, 16, 9), (3, 40, 16, 90), (7, 33, 32, 200), (64, 20, 64, 1500), (300, 70, 16, 9000), (1100, 9, 16, 5000), (2, 900, 16, 70000), (8192, 3, 16, 9000), (3, 7, 16, 700001)])
def test_pages_advance(seqs, width, page, n_pages):
    rng = random.Random(seqs * width)
    for window, sinks in ((0, 0), (1, 0), (page, 1), (3 * page + 5, page + 1), (10 ** 9, 4)):
        table, lens, refs = state(rng, seqs, width, page, n_pages)
        new = [rng.choice([0, 1, 2, page, 3 * page + 1]) for _ in lens]
        if rng.random() < 0.8:
            new = [min(n, width * page - m) for n, m in zip(new, lens)]
        want = ref.advance(table, lens, refs, new, page, window, sinks)
        a = [i32(x) for x in (table, lens, refs, new)]
        outs = [torch.full_like(x, 77) for x in a[:3]] + [i32([77])]
        pages_advance(*a, *outs, page_size=page, window=window, sinks=sinks)
        assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[3]]]
        assert [x.tolist() for x in a] == [table, lens, refs, new]
        pages_advance(*a, *a[:3], outs[3], page_size=page, window=window, sinks=sinks)  # in place
        assert [x.tolist() for x in a[:3]] + [outs[3].item()] == [want[0], want[1], want[2], want[3]]


def test_pages_advance_says_when_there_are_too_few_pages():
    a = [i32(x) for x in ([[0, -1, -1], [1, 2, -1]], [16, 30], [1, 1, 1, 0, 0], [33, 3])]
    outs = [torch.full_like(x, 77) for x in a[:3]] + [i32([77])]
    pages_advance(*a, *outs, page_size=16)
    assert outs[3].item() == -4 and all(torch.equal(x, y) for x, y in zip(a, outs[:3]))
    for new, code in (([32, 2], 0), ([48, 0], -4), ([0, -1], -1)):  # (just enough; a row that is too long; no number of positions)
        a[3] = i32(new)
        pages_advance(*a, *outs, page_size=16)
        assert outs[3].item() == code
    a[1] = i32([49, 0])
    pages_advance(*a, *outs, page_size=16)
    assert outs[3].item() == -1


@pytest.mark.parametrize("seqs,width,page,n_pages,layers,hkv,dh,dtype", [
    (1, 3, 16, 4, 1, 1, 64, BF), (4, 12, 16, 90, 3, 2, 64, BF), (9, 7, 32, 120, 2, 1, 128, F16), (65, 9, 16, 900, 2, 8, 128, BF), (40, 4, 64, 300, 1, 3, 64, F16), (1500, 3, 16, 7000, 1, 1, 64, BF), (8192, 2, 16, 9000, 1, 1, 64, BF)])
def test_pages_reorder(seqs, width, page, n_pages, layers, hkv, dh, dtype):
    rng = random.Random(seqs)
    for kind in ("beams", "identity", "all of one", "ends", "reversed"):
        table, lens, refs = state(rng, seqs, width, page, n_pages)
        refs = [r + (rng.random() < 0.02) for r in refs]  # (pages that somebody else holds)
        parents = {"beams": [rng.randrange(-1, seqs) for _ in range(seqs)], "identity": list(range(seqs)), "all of one": [rng.randrange(seqs)] * seqs,
                   "ends": [s if rng.random() < 0.5 else -1 for s in range(seqs)], "reversed": list(range(seqs))[::-1]}[kind]
        want = ref.reorder(table, lens, refs, parents, page)
        pool = torch.randn(layers, n_pages, 2, hkv, page, dh, device="cuda").to(dtype)
        want_pool = pool.clone()
        for src, dst, fill in want[3]:
            want_pool[:, dst, :, :, :fill] = want_pool[:, src, :, :, :fill]
        a = [i32(x) for x in (table, lens, refs, parents)]
        outs, copies = [torch.full_like(x, 77) for x in a[:3]] + [i32([77])], torch.empty(1 + 3 * seqs, dtype=torch.int32, device="cuda")
        pages_reorder(pool, *a, *outs, copies=copies)
        assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[4]]], kind
        n = copies[0].item()
        assert [tuple(x) for x in copies[1:1 + 3 * n].view(-1, 3).tolist()] == want[3]
        assert torch.equal(pool, want_pool), kind
        assert [x.tolist() for x in a] == [table, lens, refs, parents]


def test_pages_reorder_refuses_on_the_device():
    pool = torch.randn(1, 4, 2, 1, 16, 64, device="cuda").to(BF)
    before = pool.clone()
    # no page for the second child's last page; a parent out of range; a length out of range; a page out of range
    for table, lens, refs, parents, code in (
            ([[0, 1], [2, -1]], [20, 3], [1, 1, 1, 1], [0, 0], 0), ([[0, 1], [2, 3]], [20, 20], [2, 2, 1, 1], [0, 0], 0),
            ([[0, 1], [2, 3]], [20, 20], [2, 2, 2, 2], [0, 0], -4), ([[0, 1], [2, 3]], [20, 20], [1, 1, 1, 1], [0, 2], -1),
            ([[0, 1], [2, 3]], [20, 20], [1, 1, 1, 1], [0, -2], -1), ([[0, 1], [2, 3]], [20, 33], [1, 1, 1, 1], [0, 0], -1),
            ([[0, 1], [2, 4]], [20, 20], [1, 1, 1, 1], [1, 0], -1)):
        a = [i32(x) for x in (table, lens, refs, parents)]
        outs = [torch.full_like(x, 77) for x in a[:3]] + [i32([77])]
        pages_reorder(pool, *a, *outs)
        assert outs[3].item() == code, (table, parents)
        if code:
            assert all(torch.equal(x, y) for x, y in zip(a, outs[:3])) and torch.equal(pool, before)
        else:
            assert outs[0].tolist()[0] == table[0] and outs[1].tolist() == [20, 20]
            pool.copy_(before)


@pytest.mark.parametrize("n_pages,layers,hkv,dh,page,dtype", [(1, 1, 1, 64, 16, BF), (2, 2, 1, 64, 16, BF), (50, 3, 2, 128, 16, F16), (333, 2, 1, 64, 64, BF), (1025, 1, 8, 128, 16, BF), (5000, 1, 1, 64, 32, F16)])
def test_pages_compact(n_pages, layers, hkv, dh, page, dtype):
    rng = random.Random(n_pages)
    for share in (0.0, 0.03, 0.5, 0.9, 1.0):
        refs = [rng.randint(1, 3) if rng.random() < share else 0 for _ in range(n_pages)]
        used = [p for p, r in enumerate(refs) if r]
        table = [[rng.choice(used) if used and rng.random() < 0.8 else -1 for _ in range(17)] for _ in range(5)]
        table[0][0] = n_pages
        want = ref.compact(table, refs)
        pool = torch.randn(layers, n_pages, 2, hkv, page, dh, device="cuda").to(dtype)
        want_pool = pool.clone()
        for src, dst in want[4]:
            want_pool[:, dst] = pool[:, src]
        a = [i32(x) for x in (table, refs)]
        outs = [torch.full_like(x, 77) for x in (a[0], a[1], a[1])] + [i32([77])]
        moves = torch.empty(1 + n_pages, dtype=torch.int32, device="cuda")
        pages_compact(pool, *a, *outs, moves=moves)
        assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[3]]]
        m, half = moves.tolist(), 1 + n_pages // 2
        assert list(zip(m[half:half + m[0]], m[1:1 + m[0]])) == want[4]
        assert torch.equal(pool, want_pool)
        pages_compact(pool, *a, a[0], a[1], *outs[2:])  # in place (the values move once more, to the same places)
        assert [x.tolist() for x in a] == [want[0], want[1]] and torch.equal(pool, want_pool)


# ---------------------------------------------------------------- streams, graphs, all of it together
def test_on_another_stream_and_in_a_graph():
    pool, table, lens = ref.cache([300, 40], 16, 2, 128, BF, 9)
    for new in (1, 100):
        q = torch.randn(new, 8, 128, device="cuda").to(BF)
        want = torch.empty_like(q)
        args = (i32([0, new, new]), pool, 1, table, lens)
        window_attention(q, want, *args, window=90, sinks=4, max_q=new)
        out, st = torch.zeros_like(q), torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        window_attention(q, out, *args, window=90, sinks=4, max_q=new, stream=st)
        st.synchronize()
        assert torch.equal(out, want)
        out.zero_()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            window_attention(q, out, *args, window=90, sinks=4, max_q=new)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_moving_pages_in_a_graph_and_on_another_stream():
    """Both kernels of a call, the second one under programmatic launch."""
    rng = random.Random(5)
    n, seqs = 300, 40
    table, lens, refs = state(rng, seqs, 6, 16, n)
    parents = [rng.randrange(seqs) for _ in range(seqs)]
    pool0 = torch.randn(8, n, 2, 8, 16, 64, device="cuda").to(BF)
    want = ref.reorder(table, lens, refs, parents, 16)
    want_pool = pool0.clone()
    for src, dst, fill in want[3]:
        want_pool[:, dst, :, :, :fill] = pool0[:, src, :, :, :fill]
    after = ref.compact(want[0], want[2])
    for src, dst in after[4]:
        want_pool[:, dst] = want_pool[:, src].clone()
    pool = pool0.clone()
    a = [i32(x) for x in (table, lens, refs, parents)]
    outs, ends = [torch.empty_like(x) for x in a[:3]] + [i32([77])], [torch.empty_like(x) for x in (a[0], a[2], a[2])] + [i32([77])]

    def both(stream=None):
        pages_reorder(pool, *a, *outs, stream=stream)
        pages_compact(pool, outs[0], outs[2], *ends, stream=stream)

    def check():
        assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [0]]
        assert [x.tolist() for x in ends] == [after[0], after[1], after[2], [after[3]]]
        assert torch.equal(pool, want_pool)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    both(st)
    st.synchronize()
    check()
    pool.copy_(pool0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(2):
        pool.copy_(pool0)
        g.replay()
        torch.cuda.synchronize()
        check()


def test_pages_in_a_graph():
    a = [i32(x) for x in ([[0, -1, -1, -1], [1, 2, -1, -1]], [16, 30], [1, 1, 1, 0, 0, 0, 0, 0], [1, 1])]
    outs = [torch.empty_like(x) for x in a[:3]] + [i32([77])]
    pool = torch.randn(1, 8, 2, 1, 16, 64, device="cuda").to(BF)
    r_outs = [torch.empty_like(x) for x in a[:3]] + [i32([77])]
    par = i32([1, 1])
    pages_reorder(pool, *outs[:3], par, *r_outs)  # (first use outside the capture)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pages_advance(*a, *outs, page_size=16)
        pages_reorder(pool, *outs[:3], par, *r_outs)
    g.replay()
    torch.cuda.synchronize()
    assert outs[0].tolist() == [[0, 3, -1, -1], [1, 2, -1, -1]] and outs[1].tolist() == [17, 31] and outs[3].item() == 0
    want = ref.reorder(outs[0].tolist(), outs[1].tolist(), outs[2].tolist(), [1, 1], 16)
    assert [x.tolist() for x in r_outs] == [want[0], want[1], want[2], [0]]

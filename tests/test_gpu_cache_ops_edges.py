"""The operators on a caller's paged cache at their ends: calls without tokens, threads, errors left by others, small probabilities and infinities
in f16, status words, lengths and starts that cannot be, and launches that only large or unaligned calls take (needs a B200)."""
import ctypes as C
import importlib.util
import os
import random
import threading

import pytest
import torch

from paper_2604_18396_b200 import binding, cache_ops, pages_advance, pages_compact, pages_reorder, rope_append, window_attention
from tests import paged_reference as ref
from tests import test_gpu_cache_ops as base

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def freq(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


# ---------------------------------------------------------------- calls without tokens
def test_empty_tensors_are_no_tokens():
    """An idle step: torch gives tensors without elements the address 0."""
    pool, table, lens = ref.cache([20], 16, 2, 64, BF, 1)
    before, status = pool.clone(), i32([0])
    rows = lambda h: torch.empty(0, h, 64, dtype=BF, device="cuda")  # noqa: E731
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert rows(2).data_ptr() == 0
    rope_append(rows(4), rows(2), rows(2), none, none, freq(64), pool, 1, table, rows(4), status=status)
    rope_append(None, rows(2), rows(2), none, none, freq(64), pool, 1, table, None, status=status)
    for max_q in (0, 1):
        window_attention(rows(4), rows(4), i32([0, 0]), pool, 1, table, lens, window=8, max_q=max_q, status=status)
    assert status.item() == 0 and torch.equal(pool.view(torch.int16), before.view(torch.int16))


# ---------------------------------------------------------------- threads and errors of others
def test_reorderings_of_several_threads():
    """Calls that need different amounts of shared memory, side by side."""
    lib, failures = binding.load(), []

    def work(seqs):
        st = torch.cuda.Stream()
        pool = torch.zeros(1, 1, 2, 1, 16, 64, dtype=BF, device="cuda")
        a = [torch.full((seqs, 1), -1, dtype=torch.int32, device="cuda"), i32([0] * seqs), i32([0]), i32([-1] * seqs)]
        outs = [torch.empty_like(x) for x in a[:3]] + [torch.empty(1 + 3 * seqs, dtype=torch.int32, device="cuda"), i32([77])]
        torch.cuda.synchronize()
        cache = cache_ops._PAGED.pack(pool.data_ptr(), a[0].data_ptr(), a[1].data_ptr(), 0, 1, 1, 1, 64, 16, seqs, 1)
        args = (cache, a[2].data_ptr(), a[3].data_ptr(), *(x.data_ptr() for x in outs), st.cuda_stream)
        codes = {lib.river_pages_reorder(*args) for _ in range(20000)}
        st.synchronize()
        if codes != {0} or outs[4].item():
            failures.append((seqs, codes))

    threads = [threading.Thread(target=work, args=(n,)) for n in (8192, 2048, 8192, 2048)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures


def test_a_launch_that_failed_is_not_the_next_calls_error():
    """A launch into a capture that has been broken off is refused; calls on other streams know nothing of it."""
    cu, lib = C.CDLL("libcuda.so.1"), binding.load()
    st = torch.cuda.Stream()
    handle, graph = C.c_void_p(st.cuda_stream), C.c_void_p()
    a = [i32([[0, -1]]), i32([3]), i32([1, 0]), i32([1])]
    outs = [torch.empty_like(x) for x in a[:3]] + [i32([77])]
    k, q = torch.randn(1, 2, 64, device="cuda").to(BF), torch.randn(1, 2, 64, device="cuda").to(BF)
    out, zero, f, start = torch.empty_like(q), i32([0]), freq(64), i32([0, 1])
    par, reordered = i32([0]), [torch.empty_like(x) for x in a[:3]] + [i32([77])]
    copies = torch.empty(4, dtype=torch.int32, device="cuda")
    p2 = torch.zeros(1, 2, 2, 2, 16, 64, dtype=BF, device="cuda")
    c_adv = cache_ops._PAGED.pack(0, a[0].data_ptr(), a[1].data_ptr(), 0, 1, 2, 1, 64, 16, 1, 2)
    c_pool = cache_ops._PAGED.pack(p2.data_ptr(), a[0].data_ptr(), a[1].data_ptr(), 0, 1, 2, 2, 64, 16, 1, 2)
    calls = {
        "advance": lambda s: lib.river_pages_advance(c_adv, a[2].data_ptr(), a[3].data_ptr(), 0, 0, *(x.data_ptr() for x in outs), s),
        "reorder": lambda s: lib.river_pages_reorder(c_pool, a[2].data_ptr(), par.data_ptr(), *(x.data_ptr() for x in reordered[:3]), copies.data_ptr(), reordered[3].data_ptr(), s),
        "rope": lambda s: lib.river_rope_append(c_pool, 1, 1, 0, 0, None, cache_ops._rows(k, 0, "k"), cache_ops._rows(k, 0, "v"), zero.data_ptr(), zero.data_ptr(), f.data_ptr(), 64, 0, 1.0, 0, 0, s),
        "attention": lambda s: lib.river_window_attention(c_pool, 1, 1, 1, start.data_ptr(), 2, cache_ops._rows(q, 0, "q"), 8, 0, 0.125, out.data_ptr(), 0, s),
    }
    torch.cuda.synchronize()
    for name, call in calls.items():
        assert cu.cuStreamBeginCapture_v2(handle, 2) == 0
        assert cu.cuStreamSynchronize(handle) != 0  # (not allowed: the capture is invalid from here on)
        assert call(st.cuda_stream) == -6, name
        assert cu.cuStreamEndCapture(handle, C.byref(graph)) != 0
        for other in calls.values():
            assert other(0) == 0, name
    torch.cuda.synchronize()


# ---------------------------------------------------------------- a wait that runs out
@pytest.mark.parametrize("splits", [1, 2, 4])
@pytest.mark.parametrize("dtype,dh", [(BF, 128), (F16, 64)])
def test_a_wait_that_runs_out_stores_no_row(splits, dtype, dh):
    """CTAs that never ask for their keys: their waits end, the status says so, and no row of their clusters is stored."""
    lib, hq, hkv = binding.load(), 4, 2
    pool, table, lens = ref.cache([600, 300], 16, hkv, dh, dtype, 7)
    q = torch.randn(300, hq, dh, generator=torch.Generator().manual_seed(8)).to(dtype).cuda()
    starts = [0, 200, 300]
    want, tol = ref.attention(q, starts, pool, 1, table, [600, 300], 400, 4, 0.125)
    cache, q_start = cache_ops._PAGED.pack(pool.data_ptr(), table.data_ptr(), lens.data_ptr(), cache_ops._TYPES[dtype], 1, pool.shape[1], hkv, dh, 16, 2, table.shape[1]), i32(starts)
    for status in (i32([0]), None):
        out = torch.full_like(q, NAN)
        rc = lib.river_selftest_window_timeout(cache, 1, 300, 200, q_start.data_ptr(), hq, cache_ops._rows(q, 0, "q"), 400, 4, 0.125, out.data_ptr(),
                                               status.data_ptr() if status is not None else 0, splits, 2000, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == 0 and (status is None or status.item() == -7)
        assert out[:, :2].isnan().all() and ((out.double() - want).abs() <= tol)[:, 2:].all()
    out, status = torch.full_like(q, NAN), i32([0])  # and the kernel is none the worse for it
    window_attention(q, out, q_start, pool, 1, table, lens, window=400, sinks=4, max_q=200, softmax_scale=0.125, status=status)
    assert status.item() == 0 and ((out.double() - want).abs() <= tol).all()


# ---------------------------------------------------------------- f16
@pytest.mark.parametrize("new", [1, 64])
def test_f16_many_weak_positions_beside_a_strong_one(new):
    """32768 positions of 2^-25 each of the strongest weigh 2^-10 together.  A probability is kept to 2^-24 of the largest that the type
    has room for: 2^-24 / 2^15 (single tokens), 2^-24 / 2^7 (prompts)."""
    n, dh, page = 32768 + new, 64, 64
    pool, table, lens = ref.cache([n], page, 1, dh, F16, 3, fill=0.0)
    pool[:, :, 0], pool[:, :, 1] = 0.0, 1.0
    first = table[0, 0].long()
    pool[0, first, 0, 0, 0], pool[0, first, 1, 0, 0] = 2.175, 0.0
    q = torch.ones(new, 2, dh, dtype=F16, device="cuda")
    out, status = torch.full_like(q, NAN), i32([0])
    window_attention(q, out, i32([0, new]), pool, 1, table, lens, window=n, max_q=new, status=status)
    want, _ = ref.attention(q, [0, new], pool, 1, table, [n], n, 0, dh ** -0.5)
    assert status.item() == 0 and 5e-4 < want.min().item() and want.max().item() < 2e-3
    fp32 = 2 * (dh + 8) * 2.0 ** -24 * 64 * 2.175 / 8 + (n + 8) * 2.0 ** -23
    tol = ref.U[F16] * want + fp32 * want + n * 2.0 ** -24 * 2.0 ** (-15 if new == 1 else -7) + ref.TINY[F16]
    assert ((out.double() - want).abs() <= tol).all(), ((out.double() - want).abs() / tol).max().item()


@pytest.mark.parametrize("dtype", [F16, BF])
@pytest.mark.parametrize("new", [1, 64, 300])
def test_scores_of_many_millions(new, dtype):
    """However coarse a float is at the scores' size, every probability is a number."""
    n, dh, page = 700, 128, 16
    pool, table, lens = ref.cache([n], page, 1, dh, dtype, 3, fill=0.0)
    q = torch.ones(new, 2, dh, dtype=dtype, device="cuda")
    q[:, 1] *= -1
    for x in (500.0, 1000.0, 1901.0, 3001.0, 7777.0, 20000.0, 65000.0) + ((1e6, 1e9, 1e12) if dtype is BF else ()):
        pool[:, :, 0] = -x
        pool[0, table[0, 0].long(), 0, 0, 5] = x
        pool[0, table[0, 20].long(), 0, 0, 3] = x
        out = torch.full_like(q, NAN)
        window_attention(q * x, out, i32([0, new]), pool, 1, table, lens, window=n, max_q=new)
        want, tol = ref.attention(q * x, [0, new], pool, 1, table, [n], n, 0, dh ** -0.5)
        assert ((out.double() - want).abs() <= tol).all(), x


@pytest.mark.parametrize("dtype", [F16, BF])
@pytest.mark.parametrize("n,new,j", [(1000, 1, 5), (1000, 3, 13), (1000, 1, 200), (1000, 64, 200), (1000, 64, 990), (1000, 200, 3), (1000, 200, 850), (400, 380, 15), (400, 380, 90)])
@pytest.mark.parametrize("value", [INF, -INF])
def test_an_infinite_value_behind_a_small_probability(n, new, j, value, dtype):
    """Far below the smallest number of 16 bits, but a number in 32: the result is infinite where the position is seen, and only there."""
    dh, page, dim = 128, 16, 7
    pool, table, lens = ref.cache([n], page, 2, dh, dtype, 3, fill=0.0)
    pool[:, :, 0] = 0.0
    pool[0, table[0, 0].long(), 0, :, 0] = 2.65  # q k / sqrt(dh) = 30: the others have 2^-43 of its weight
    q = torch.ones(new, 4, dh, dtype=dtype, device="cuda")
    want, tol = ref.attention(q, [0, new], pool, 1, table, [n], n, 0, dh ** -0.5)
    pool[0, table[0, j // page].long(), 1, 1, j % page, dim] = value
    out, status = torch.full_like(q, NAN), i32([0])
    window_attention(q, out, i32([0, new]), pool, 1, table, lens, window=n, max_q=new, status=status)
    sees = torch.arange(n - new, n, device="cuda") >= j
    assert status.item() == 0
    assert (out[sees][:, 2:, dim] == value).all()
    same = (out.double() - want).abs() <= tol
    same[sees, 2:, dim] = True
    assert same.all()


@pytest.mark.parametrize("dtype", [F16, BF])
@pytest.mark.parametrize("new,j", [(1, 5), (3, 199), (100, 20), (300, 350)])
def test_a_key_that_is_no_number_is_none_in_the_result(new, j, dtype):
    n, dh = 400, 64
    pool, table, lens = ref.cache([n], 16, 2, dh, dtype, 3, fill=0.0)
    q = torch.randn(new, 4, dh, generator=torch.Generator().manual_seed(8)).to(dtype).cuda()
    want, tol = ref.attention(q, [0, new], pool, 1, table, [n], n, 0, dh ** -0.5)
    pool[0, table[0, j // 16].long(), 0, 1, j % 16, 7] = NAN
    out = torch.full_like(q, 0.0)
    window_attention(q, out, i32([0, new]), pool, 1, table, lens, window=n, max_q=new)
    sees = torch.arange(n - new, n, device="cuda") >= j
    assert out[sees][:, 2:].isnan().all()
    same = (out.double() - want).abs() <= tol
    same[sees, 2:] = True
    assert same.all()


# ---------------------------------------------------------------- what is told
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("inter", [True, False])
def test_rope_append_tells_sequences_below_padding(aligned, inter):
    pool, table, _ = ref.cache([40, 20], 16, 2, 64, BF, 3, fill=0.0)
    before = pool.clone()
    x = torch.randn(1 + 2 * 8 * 64, device="cuda").to(BF)
    x = (x[:-1] if aligned else x[1:]).view(2, 8, 64)
    q, k, v = x.split([4, 2, 2], 1)
    for bad in (-2, -2 ** 31):
        q_out, status = torch.full((2, 4, 64), NAN, dtype=BF, device="cuda"), i32([0])
        rope_append(q, k, v, i32([5, 6]), i32([-1, bad]), freq(64), pool, 1, table, q_out, interleaved=inter, status=status)
        assert status.item() == -1 and torch.equal(pool, before)
        want = ref.rope(q[1:], i32([6]), freq(64), inter, 1.0)
        assert (q_out[0] == 0).all() and ((q_out[1:].double() - want).abs() <= ref.U[BF] * want.abs() + 2.0 ** -19 * q.abs().max()).all()


def test_window_attention_answers_the_first_max_q_queries():
    """A sequence with more queries than max_q is told, and its first max_q rows are right."""
    pool, table, lens = ref.cache([50, 40], 16, 1, 64, BF, 4)
    q = torch.randn(5, 2, 64, device="cuda").to(BF)
    for max_q in (1, 2, 3):
        out, status = torch.zeros_like(q), i32([0])
        window_attention(q, out, i32([0, 4, 5]), pool, 1, table, lens, window=10, sinks=2, max_q=max_q, status=status)
        want, tol = ref.attention(q, [0, 4, 5], pool, 1, table, [50, 40], 10, 2, 0.125)
        rows = list(range(max_q)) + [4]
        assert status.item() == -1 and ((out.double() - want).abs() <= tol)[rows].all(), max_q


@pytest.mark.parametrize("tokens,beams,steps,pages", [(90, 1, 20, 6), (300, 2, 6, 5), (64, 4, 30, 9)])
def test_the_example_ends_with_an_error_where_pages_do_not_suffice(tokens, beams, steps, pages):
    root = os.path.dirname(os.path.dirname(os.path.abspath(base.__file__)))
    spec = importlib.util.spec_from_file_location("windowed_beams", os.path.join(root, "examples", "windowed_beams.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    prompt = torch.randint(0, ex.VOCAB, (tokens,), generator=torch.Generator().manual_seed(2)).cuda()
    with pytest.raises(RuntimeError):
        ex.run(ex.Model(), prompt, beams=beams, steps=steps, window=1000, sinks=0, pages=pages)


@pytest.mark.parametrize("bad", [-5, -1, -2 ** 31, -2 ** 31 + 1])
@pytest.mark.parametrize("new", [1, 40])
def test_window_attention_tells_negative_lengths(new, bad):
    """Such a sequence holds nothing; the others are as ever."""
    pool, table, lens = ref.cache([60, 70], 16, 1, 64, BF, 4)
    q = torch.randn(2 * new, 2, 64, device="cuda").to(BF)
    out, status = torch.full_like(q, NAN), i32([0])
    window_attention(q, out, i32([0, new, 2 * new]), pool, 1, table, i32([bad, 70]), window=20, sinks=2, max_q=new, status=status)
    want, tol = ref.attention(q, [0, new, 2 * new], pool, 1, table, [0, 70], 20, 2, 0.125)
    assert status.item() == -1 and (out[:new] == 0).all() and ((out.double() - want).abs() <= tol).all()
    status.zero_()  # (a sequence without queries may have any)
    window_attention(q[:new], out[:new], i32([0, 0, new]), pool, 1, table, i32([bad, 70]), window=20, sinks=2, max_q=new, status=status)
    want, tol = ref.attention(q[:new], [0, 0, new], pool, 1, table, [0, 70], 20, 2, 0.125)
    assert status.item() == 0 and ((out[:new].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("hq", [4, 256])  # (256 heads to two: a tile for every query)
@pytest.mark.parametrize("starts", [[0, 5, -2 ** 31], [0, 2 ** 31 - 1, 80], [2 ** 31 - 1, 3, 80], [-2 ** 31, 3, 80], [0, 81, 80], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1],
                                    [-1, -2 ** 31, 80], [7, 2 ** 31 - 2, -2 ** 31 + 5]])
def test_window_attention_tells_starts_that_cannot_be(starts, hq):
    """Whatever stands there: it is told, and no row but those of sound sequences is written."""
    pool, table, lens = ref.cache([90, 100], 16, 2, 64, BF, 4)
    q = torch.randn(80, hq, 64, device="cuda").to(BF)
    for max_q in (1, 80):
        around, status = torch.full((3 * 80, hq, 64), NAN, dtype=BF, device="cuda"), i32([0])
        out = around[80:160]
        window_attention(q, out, i32(starts), pool, 1, table, lens, window=20, sinks=2, max_q=max_q, status=status)
        assert status.item() == -1 and around[:80].isnan().all() and around[160:].isnan().all()
        for s, n in enumerate((90, 100)):
            a, b = starts[s], starts[s + 1]
            if 0 <= a <= b <= 80:
                b = min(b, a + max_q)
                want, tol = ref.attention(q[a:b], [0, b - a], pool, 1, table[s:s + 1], [n - (starts[s + 1] - b)], 20, 2, 0.125)
                assert ((out[a:b].double() - want).abs() <= tol).all()
                around[80 + a:80 + starts[s + 1]] = NAN
        assert around.isnan().all()


def test_pages_advance_wants_more_pages_than_32_bits_count():
    """8192 sequences that want 262145 pages each, and 524288: 2^31 and 2^32 and a few more."""
    seqs, page = 8192, 16
    for width in (262145, 524289):
        table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
        lens, refs, status = torch.zeros(seqs, dtype=torch.int32, device="cuda"), torch.zeros(50000, dtype=torch.int32, device="cuda"), i32([77])
        pages_advance(table, lens, refs, torch.full_like(lens, width * page), table, lens, refs, status, page_size=page)
        assert status.item() == -4 and not lens.any() and not refs.any() and table[0, 0].item() == -1 and table.max().item() == -1
        pages_advance(table, lens, refs, torch.full_like(lens, 96), table, lens, refs, status, page_size=page)  # 49152 pages
        assert status.item() == 0 and (lens == 96).all() and (refs[:49152] == 1).all() and not refs[49152:].any()
        assert torch.equal(table[:, :6].flatten(), torch.arange(49152, dtype=torch.int32, device="cuda")) and table[:, 6:].max().item() == -1
        del table


def test_steps_of_one_token_and_one_head_may_be_anything():
    """A view of one row that is 3 longer than its heads, and one head of rows of any length."""
    pool, table, lens = ref.cache([50], 16, 1, 64, BF, 4)
    row = torch.randn(1, 4 * 64 + 3, device="cuda").to(BF)
    q = row.as_strided((1, 4, 64), (259, 64, 1))
    heads = torch.randn(64 * 9, device="cuda").to(BF).as_strided((9, 1, 64), (64, 7, 1))
    for x in (q, heads):
        out, status, n = torch.full(x.shape, NAN, dtype=BF, device="cuda"), i32([0]), x.shape[0]
        window_attention(x, out, i32([0, n]), pool, 1, table, lens, window=20, sinks=2, max_q=n, status=status)
        want, tol = ref.attention(x, [0, n], pool, 1, table, [50], 20, 2, 0.125)
        assert status.item() == 0 and ((out.double() - want).abs() <= tol).all()


# ---------------------------------------------------------------- launches of large and unaligned calls
@pytest.mark.parametrize("t,hq,hkv,dh,rot,inter,tin,tc,page,packed", [
    (592, 32, 8, 128, 128, False, BF, BF, 16, True), (701, 8, 2, 64, 64, False, F32, F16, 32, True), (1999, 4, 1, 64, 48, True, BF, BF, 16, True),
    (593, 1, 1, 64, 16, True, F16, F16, 64, True), (799, 24, 8, 128, 98, True, F32, BF, 16, True), (1030, 3, 1, 128, 32, False, F16, F16, 64, True),
    # rows of 16 bytes with a turned part that is none: the dims behind it go by eights
    (5, 3, 1, 128, 34, False, F16, F16, 16, True), (650, 6, 2, 128, 18, False, BF, BF, 32, True), (9, 4, 4, 128, 62, False, F32, BF, 16, True),
    (700, 2, 2, 64, 6, False, F32, F16, 64, True), (650, 5, 1, 64, 34, True, BF, BF, 16, False)])
def test_rope_append_of_prompts(t, hq, hkv, dh, rot, inter, tin, tc, page, packed):
    base.test_rope_append(t, hq, hkv, dh, rot, inter, tin, tc, page, packed)


def test_pages_reorder_of_wide_tables():
    base.test_pages_reorder(300, 900, 16, 9000, 1, 1, 64, BF)


def test_pages_compact_of_many_pages():
    base.test_pages_compact(262200, 1, 1, 64, 16, BF)


def off16(v):
    """The same ints, four bytes behind a 16-byte boundary."""
    x = i32(v)
    y = torch.empty(x.numel() + 1, dtype=torch.int32, device="cuda")[1:].view(x.shape)
    return y.copy_(x)


@pytest.mark.parametrize("seqs,width,n_pages", [(3, 7, 60), (70, 33, 3001)])
def test_pages_off_16_bytes(seqs, width, n_pages):
    rng, page = random.Random(seqs), 16
    table, lens, refs = base.state(rng, seqs, width, page, n_pages)
    new = [min(rng.choice([0, 1, page, 40]), width * page - m) for m in lens]
    want = ref.advance(table, lens, refs, new, page, 50, 3)
    a = [off16(x) for x in (table, lens, refs, new)]
    outs = [off16(x) for x in (table, lens, refs)] + [i32([77])]
    pages_advance(*a, *outs, page_size=page, window=50, sinks=3)
    assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[3]]]
    parents = [rng.randrange(-1, seqs) for _ in range(seqs)]
    want = ref.reorder(table, lens, refs, parents, page)
    pool = torch.randn(2, n_pages, 2, 1, page, 64, device="cuda").to(BF)
    want_pool = pool.clone()
    for src, dst, fill in want[3]:
        want_pool[:, dst, :, :, :fill] = want_pool[:, src, :, :, :fill]
    pages_reorder(pool, *a[:3], off16(parents), *outs)
    assert [x.tolist() for x in outs] == [want[0], want[1], want[2], [want[4]]] and torch.equal(pool, want_pool)
    want = ref.compact(table, refs)
    for src, dst in want[4]:
        want_pool[:, dst] = want_pool[:, src].clone()
    outs, n = [off16(table), off16(refs), off16(refs)], off16([77])
    pages_compact(pool, a[0], a[2], *outs, n)
    assert [x.tolist() for x in outs] + [n.item()] == [want[0], want[1], want[2], want[3]] and torch.equal(pool, want_pool)


@pytest.mark.parametrize("seqs,hq,hkv,dh,width,dtype", [(128, 32, 8, 128, 32768, BF), (48, 32, 8, 128, 131072, F16), (32, 8, 8, 128, 32768, BF), (200, 8, 1, 64, 65536, BF)])
def test_single_tokens_under_long_windows(seqs, hq, hkv, dh, width, dtype):
    """Ordinary attention of short conversations whose table has room for long ones."""
    rng = random.Random(seqs)
    lens = [rng.choice([1, 17, 300, rng.randint(1, 900)]) for _ in range(seqs)]
    pool, table, lens_t = ref.cache(lens, 16, hkv, dh, dtype, 7, width=width // 16)
    q = (torch.randn(seqs, hq, dh, generator=torch.Generator().manual_seed(8)) * 2).to(dtype).cuda()
    out, status, starts = torch.full_like(q, NAN), i32([0]), list(range(seqs + 1))
    window_attention(q, out, i32(starts), pool, 1, table, lens_t, window=width, max_q=1, status=status)
    want, tol = ref.attention(q, starts, pool, 1, table, lens, width, 0, dh ** -0.5)
    assert status.item() == 0 and ((out.double() - want).abs() <= tol).all()

"""Calls of the operators on a paged cache at their ends, as far as the host alone decides (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_18396_b200 import cache_ops
from tests import test_cache_ops_checks as checks

lib = checks.lib
NONE = (0, 256, 64)  # rows of a tensor without elements: no address


def test_calls_without_tokens_need_no_addresses(lib):
    assert checks.rope(lib, n=0, q=NONE, k=NONE, v=NONE, pos=0, seqs=0, out=0) == 0
    assert checks.attn(lib, n=0, q=NONE, out=0) == 0


@pytest.mark.parametrize("kw", [dict(layer=0), dict(rot=0), dict(f=0)])
def test_calls_without_tokens_are_checked_all_the_same(lib, kw):
    assert checks.rope(lib, n=0, q=NONE, k=NONE, v=NONE, pos=0, seqs=0, out=0, **kw) == -1
    if "layer" in kw:
        assert checks.attn(lib, n=0, q=NONE, out=0, **kw) == -1 and checks.attn(lib, n=0, q=NONE, out=0, window=0) == -1


def test_the_self_test_of_waits_refuses_what_it_cannot_run(lib):
    def call(splits=1, polls=1000, n=4, hq=4, c=None):
        return lib.river_selftest_window_timeout(C.byref(c or checks.paged()), 1, n, 2, checks.P, hq, C.byref(cache_ops.river_rows(checks.P, 256, 64)),
                                                 8, 0, 1.0, checks.P, 0, splits, polls, 0)
    assert [call(splits=x) for x in (0, 3, 8)] == [-1] * 3 and [call(polls=x) for x in (0, -1, (1 << 20) + 1)] == [-1] * 3
    assert call(n=0) == -1 and call(hq=3) == -1 and call(hq=258) == -2 and call(c=checks.paged(dh=96)) == -2


def test_steps_of_dims_with_one_place_are_none():
    x = torch.zeros(1000, dtype=torch.bfloat16)
    rows = lambda *a: cache_ops._ROWS.unpack(cache_ops._rows(x.as_strided(*a), -1, "q"))[1:]  # noqa: E731
    assert rows((1, 4, 64), (259, 64, 1)) == (0, 64) and rows((3, 1, 64), (64, 7, 1)) == (64, 0) and rows((2, 3, 64), (259, 65, 1)) == (259, 65)
    with pytest.raises(ValueError):
        rows((2, 3, 64), (256, 1, 2))


ODD = checks.P + 2  # no address of an int or a float


@pytest.mark.parametrize("call,names", [(checks.rope, ("pos", "seqs", "f")), (checks.attn, ("qs",)), (checks.advance, ("refs", "new", "t", "ln", "r", "st")),
                                        (checks.reorder, ("refs", "par", "t", "ln", "r", "copies", "st")), (checks.compact, ("refs", "t", "r", "remap", "n", "moves"))])
def test_arrays_off_their_words_are_refused(lib, call, names):
    for name in names:
        assert call(lib, **{name: ODD}) == -1, name


def test_a_status_off_its_word_is_refused(lib):
    c, rows = C.byref(checks.paged()), C.byref(cache_ops.river_rows(checks.P, 256, 64))
    assert lib.river_rope_append(c, 1, 4, 4, 0, rows, rows, rows, checks.P, checks.P, checks.P, 64, 0, 1.0, checks.P, ODD, 0) == -1
    assert lib.river_window_attention(c, 1, 4, 2, checks.P, 4, rows, 8, 0, 1.0, checks.P, ODD, 0) == -1


def test_numbers_beyond_32_bits_are_refused():
    """ctypes would hand on the lower half: a window of 2^32 + 5 as one of 5."""
    pool, table, lens = torch.zeros(1, 2, 2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q, big = torch.zeros(1, 1, 64, dtype=torch.bfloat16), 2 ** 32 + 5
    args = dict(window=4, sinks=1, max_q=1)
    for name in args:
        for x in (big, 2 ** 31, -2 ** 31 - 1):
            with pytest.raises(ValueError, match="32 bits"):
                cache_ops.window_attention(q, q, lens, pool, 1, table, lens, **{**args, name: x})
    with pytest.raises(ValueError, match="32 bits"):
        cache_ops.window_attention(q, q, lens, pool, big, table, lens, **args)
    with pytest.raises(ValueError, match="32 bits"):
        cache_ops.rope_append(q, q, q, lens, lens, torch.zeros(32), pool, big, table, q)
    for kw in (dict(page_size=big), dict(page_size=16, window=big), dict(page_size=16, sinks=big)):
        with pytest.raises(ValueError, match="32 bits"):
            cache_ops.pages_advance(table, lens, lens, lens, table, lens, lens, lens, **kw)
    with pytest.raises(ValueError, match="32 bits"):
        cache_ops.rope_frequencies(64, 1e4, "ramp", factor=4.0, original_context=2 ** 32 + 4096)
    with pytest.raises(ValueError, match="32 bits"):
        cache_ops.rope_frequencies(2 ** 32 + 64, 1e4)

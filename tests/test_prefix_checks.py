"""Refusals of the operators for requests that share prefixes, that need no GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2604_18396_b200 import cache_ops, prefix_attention_bytes
from tests.test_cache_ops_checks import BAD_CACHES, P, lib, paged  # noqa: F401


def attn(lib, c=None, layer=1, n=4, mq=2, own=0, qs=P, lead=P, shared=P, hq=4, q=(P, 256, 64), scale=1.0, out=P, work=P, size=1 << 40):
    return lib.river_prefix_attention(C.byref(c or paged()), layer, n, mq, own, qs, lead, shared, hq, C.byref(cache_ops.river_rows(*q)) if q else None, scale, out,
                                      work, size, 0, 0)


def admit(lib, c=None, refs=P, like=P, begin=P, total=P, t=2 * P, ln=2 * P, r=2 * P, new=P, st=P):
    return lib.river_pages_admit(C.byref(c or paged()), refs, like, begin, total, t, ln, r, new, st, 0)


def slots(lib, c=None, new=P, n=4, qs=P, pos=P, seqs=P, out=P, st=P):
    return lib.river_pages_slots(C.byref(c or paged()), new, n, qs, pos, seqs, out, st, 0)


def groups(lib, c=None, qs=P, least=1, lead=P, shared=P):
    return lib.river_prefix_groups(C.byref(c or paged()), qs, least, lead, shared, 0)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches(lib, kw, code):  # noqa: F811
    for call in (attn, admit, slots, groups):
        if call is not attn and kw.get("pool") == 0:
            continue  # (they touch no values)
        assert call(lib, paged(**kw)) == code, call.__name__


def test_lengths_are_needed(lib):  # noqa: F811
    for call in (attn, admit, slots, groups):
        assert call(lib, paged(lens=0)) == -1 and call(lib, paged(lens=P + 2)) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(layer=0), -1), (dict(layer=3), -1), (dict(n=-1), -1), (dict(mq=-1), -1), (dict(own=-1), -1), (dict(qs=0), -1), (dict(lead=0), -1), (dict(shared=0), -1),
    (dict(lead=P + 1), -1), (dict(shared=P + 2), -1), (dict(q=None), -1), (dict(q=(0, 256, 64)), -1), (dict(q=(P + 8, 256, 64)), -1), (dict(q=(P, 260, 64)), -1),
    (dict(q=(P, 256, 68)), -1), (dict(hq=3), -1), (dict(hq=0), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(out=0), -1), (dict(out=P + 8), -1),
    (dict(hq=1 << 20), -2), (dict(hq=258), -2), (dict(n=1 << 29, hq=4), -2), (dict(work=P + 64), -1)])
def test_prefix_attention_refusals(lib, kw, code):  # noqa: F811
    assert attn(lib, **kw) == code


def test_a_call_that_needs_a_workspace_says_so(lib):  # noqa: F811
    """64 rows whose table has room for 65536 positions, a hundred of them their own: groups, which leave parts."""
    big = dict(c=paged(n_seqs=64, max_pages=4096), n=64, mq=1, own=100, hq=8)
    need = prefix_attention_bytes(64, 64, 8, 2, 64)
    assert need > 0
    assert attn(lib, **big, work=0) == -3 and attn(lib, **big, size=need - 1) == -3


def test_sizes_without_a_kernel_need_no_bytes():
    ok = (4, 4, 8, 2, 64)
    assert prefix_attention_bytes(*ok) > 0
    for k, v in ((0, 0), (0, 8193), (1, -1), (2, 0), (2, 7), (2, 258), (3, 0), (4, 96), (1, 1 << 29)):
        a = list(ok)
        a[k] = v
        assert prefix_attention_bytes(*a) == 0, a
    with pytest.raises(ValueError):
        prefix_attention_bytes(1 << 40, 1, 1, 1, 64)


def test_calls_without_tokens_do_nothing(lib):  # noqa: F811
    assert attn(lib, n=0) == 0 and attn(lib, mq=0) == 0 and attn(lib, n=0, q=None, out=0, work=0) == 0


@pytest.mark.parametrize("kw", [dict(refs=0), dict(like=0), dict(begin=0), dict(total=0), dict(t=0), dict(ln=0), dict(r=0), dict(new=0), dict(st=0), dict(t=P), dict(ln=P),
                                dict(r=P), dict(like=P + 1), dict(new=P + 2)])
def test_pages_admit_refusals(lib, kw):  # noqa: F811
    assert admit(lib, **kw) == -1


@pytest.mark.parametrize("kw,code", [(dict(new=0), -1), (dict(n=-1), -1), (dict(qs=0), -1), (dict(pos=0), -1), (dict(seqs=0), -1), (dict(out=0), -1), (dict(out=P + 4), -1),
                                     (dict(qs=P + 2), -1), (dict(n=1 << 30), -2)])
def test_pages_slots_refusals(lib, kw, code):  # noqa: F811
    assert slots(lib, **kw) == code


@pytest.mark.parametrize("kw", [dict(qs=0), dict(least=0), dict(least=-3), dict(lead=0), dict(shared=0), dict(lead=P + 2)])
def test_prefix_groups_refusals(lib, kw):  # noqa: F811
    assert groups(lib, **kw) == -1


def test_too_many_sequences(lib):  # noqa: F811
    for call in (attn, admit, slots, groups):
        assert call(lib, paged(n_seqs=8193)) == -2


def test_the_self_test_refuses_what_it_cannot_do(lib):  # noqa: F811
    def call(way=0, mute=-1, polls=64, n=4, hq=4):
        return lib.river_selftest_prefix_attention(C.byref(paged()), 1, n, 2, P, P, P, hq, C.byref(cache_ops.river_rows(P, 256, 64)), 1.0, P, P, 1 << 40, 0, way, mute, polls, 0)

    assert call(way=-1) == -1 and call(way=4) == -1 and call(polls=0) == -1 and call(polls=(1 << 20) + 1) == -1 and call(n=0) == -1
    assert call(way=1, n=1000) == -2 and call(way=2, n=1000) == -2  # (more than two query tiles of rows to a sequence)


def test_the_binding_refuses_what_it_can_see():
    pool, table = torch.zeros(1, 2, 2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    one, q = table[0, :1], pool[0, :, 0, 0]
    for call in (lambda: cache_ops.prefix_attention(q, q, table[0], pool, 1, table, one, one, one, max_q=1),
                 lambda: cache_ops.prefix_groups(table, one, table[0], one, one, page_size=16),
                 lambda: cache_ops.pages_slots(table, one, one, table[0], one, one, one.long(), page_size=16),
                 lambda: cache_ops.pages_admit(table, one, one, one, one, one, table, one, one, one, one, page_size=16),
                 lambda: cache_ops.pages_slots(table, one, one, table[0], one, one, one.long(), page_size=1 << 40),
                 lambda: cache_ops.prefix_groups(table, one, table[0], one, one, page_size=16, least=1 << 31),
                 lambda: cache_ops.prefix_attention(q, q, table[0], pool, 1, table, one, one, one, max_q=1 << 40)):
        with pytest.raises(ValueError):
            call()

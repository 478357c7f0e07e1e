"""Refusals of the operators on a paged cache that need no GPU, and the rotary frequencies against their formulas."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2604_18396_b200 import RiverError, binding, buildlib, cache_ops, rope_frequencies

P = 1 << 20  # an aligned address that nothing reads: every call below is refused before a launch


@pytest.fixture(scope="module")
def lib():
    buildlib.build()
    return binding.load()


def paged(**kw):
    d = dict(pool=P, table=P, lens=P, dtype=0, n_layers=2, n_pages=8, Hkv=2, dh=64, page_size=16, n_seqs=3, max_pages=4)
    d.update(kw)
    return cache_ops.river_paged(*(d[n] for n, _ in cache_ops.river_paged._fields_))


BAD_CACHES = [(dict(pool=0), -1), (dict(pool=P + 64), -1), (dict(table=0), -1), (dict(table=P + 2), -1), (dict(n_layers=0), -1), (dict(n_pages=0), -1),
              (dict(Hkv=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1), (dict(dtype=2), -2), (dict(dtype=-1), -2), (dict(dh=96), -2),
              (dict(page_size=8), -2), (dict(page_size=24), -2), (dict(max_pages=1 << 28), -2), (dict(n_seqs=1 << 21), -2), (dict(Hkv=2048), -2)]


def rope(lib, c=None, layer=1, n=4, hq=4, dt=0, q=(P, 256, 64), k=(P, 128, 64), v=(P, 128, 64), pos=P, seqs=P, f=P, rot=64, scale=1.0, out=P):
    rows = [C.byref(cache_ops.river_rows(*r)) if r else None for r in (q, k, v)]
    return lib.river_rope_append(C.byref(c or paged()), layer, n, hq, dt, *rows, pos, seqs, f, rot, 0, scale, out, 0, 0)


def attn(lib, c=None, layer=1, n=4, mq=2, qs=P, hq=4, q=(P, 256, 64), window=8, sinks=0, scale=1.0, out=P):
    return lib.river_window_attention(C.byref(c or paged()), layer, n, mq, qs, hq, C.byref(cache_ops.river_rows(*q)) if q else None, window, sinks, scale, out, 0, 0)


def advance(lib, c=None, refs=P, new=P, window=8, sinks=0, t=P, ln=P, r=P, st=P):
    return lib.river_pages_advance(C.byref(c or paged()), refs, new, window, sinks, t, ln, r, st, 0)


def reorder(lib, c=None, refs=P, par=P, t=2 * P, ln=2 * P, r=2 * P, copies=P, st=P):
    return lib.river_pages_reorder(C.byref(c or paged()), refs, par, t, ln, r, copies, st, 0)


def compact(lib, c=None, refs=P, t=P, r=P, remap=P, n=P, moves=P):
    return lib.river_pages_compact(C.byref(c or paged()), refs, t, r, remap, n, moves, 0)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches(lib, kw, code):
    for call in (rope, attn, reorder, compact, advance):
        if call is advance and kw.get("pool") == 0:
            continue  # (it touches no values)
        assert call(lib, paged(**kw)) == code, call.__name__


def test_lengths_are_needed_where_they_are_read(lib):
    for call in (attn, advance, reorder):
        assert call(lib, paged(lens=0)) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(layer=0), -1), (dict(layer=3), -1), (dict(n=-1), -1), (dict(hq=-1), -1), (dict(pos=0), -1), (dict(seqs=0), -1), (dict(f=0), -1), (dict(rot=0), -1),
    (dict(rot=63), -1), (dict(rot=66), -1), (dict(scale=math.inf), -1), (dict(scale=math.nan), -1), (dict(dt=1), -2), (dict(dt=3), -2), (dict(q=None), -1),
    (dict(q=(0, 1, 1)), -1), (dict(k=None), -1), (dict(v=(0, 1, 1)), -1), (dict(out=0), -1), (dict(out=P + 8), -1), (dict(k=(P + 1, 128, 64)), -1),
    (dict(dt=2, v=(P + 2, 128, 64)), -1)])
def test_rope_append_refusals(lib, kw, code):
    assert rope(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=0), -1), (dict(layer=3), -1), (dict(n=-1), -1), (dict(mq=-1), -1), (dict(qs=0), -1), (dict(q=None), -1), (dict(q=(0, 256, 64)), -1),
    (dict(q=(P + 8, 256, 64)), -1), (dict(q=(P, 260, 64)), -1), (dict(q=(P, 256, 68)), -1), (dict(window=0), -1), (dict(window=-5), -1), (dict(sinks=-1), -1),
    (dict(hq=3), -1), (dict(hq=0), -1), (dict(scale=math.nan), -1), (dict(out=0), -1), (dict(out=P + 8), -1), (dict(hq=1 << 20), -2)])
def test_window_attention_refusals(lib, kw, code):
    assert attn(lib, **kw) == code


def test_calls_without_tokens_do_nothing(lib):
    assert rope(lib, n=0) == 0 and attn(lib, n=0) == 0 and attn(lib, mq=0) == 0


@pytest.mark.parametrize("kw", [dict(refs=0), dict(new=0), dict(window=-1), dict(sinks=-1), dict(t=0), dict(ln=0), dict(r=0), dict(st=0)])
def test_pages_advance_refusals(lib, kw):
    assert advance(lib, **kw) == -1


@pytest.mark.parametrize("kw", [dict(refs=0), dict(par=0), dict(t=0), dict(ln=0), dict(r=0), dict(copies=0), dict(st=0), dict(t=P), dict(ln=P), dict(r=P)])
def test_pages_reorder_refusals(lib, kw):
    assert reorder(lib, **kw) == -1


@pytest.mark.parametrize("kw", [dict(refs=0), dict(t=0), dict(r=0), dict(remap=0), dict(n=0), dict(moves=0)])
def test_pages_compact_refusals(lib, kw):
    assert compact(lib, **kw) == -1


def test_too_many_sequences_for_the_pages(lib):
    assert advance(lib, paged(n_seqs=8193)) == -2 and reorder(lib, paged(n_seqs=8193)) == -2


def test_the_binding_refuses_what_it_can_see():
    pool, table = torch.zeros(1, 2, 2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):  # no CUDA tensors
        cache_ops.window_attention(pool[0, :, 0, 0], pool[0, :, 0, 0], table[0], pool, 1, table, table[0], window=4, max_q=1)
    with pytest.raises(ValueError):
        cache_ops.pages_advance(table, table[0], table[0], table[0], table, table[0], table[0], table[0], page_size=16)
    with pytest.raises(ValueError):
        rope_frequencies(64, 10000.0, "unheard of")
    with pytest.raises(ValueError):
        rope_frequencies(64, 10000.0, "per_pair", pair_factors=[1.0] * 31)


# ---------------------------------------------------------------- frequencies
def test_plain_and_linear_frequencies(lib):
    f, c = rope_frequencies(128, 500000.0)
    want = 500000.0 ** (-np.arange(0, 128, 2) / 128)
    assert f.dtype == torch.float32 and c == 1.0 and np.array_equal(f.numpy(), want.astype(np.float32))
    g, c = rope_frequencies(128, 500000.0, "linear", factor=4.0)
    assert c == 1.0 and np.allclose(g.numpy(), want / 4, rtol=1e-7)
    g, c = rope_frequencies(128, 500000.0, "linear", factor=4.0, attn_scale=1.5)
    assert c == 1.5


def test_frequencies_by_parts(lib):
    theta, r, ctx, factor, lo, hi = 500000.0, 128, 8192, 8.0, 1.0, 4.0
    f, c = rope_frequencies(r, theta, "by_parts", factor=factor, original_context=ctx, low_freq=lo, high_freq=hi)
    kinds = set()
    for i in range(r // 2):
        w = theta ** (-2 * i / r)
        length = 2 * math.pi / w
        if length < ctx / hi:
            want = w
            kinds.add("kept")
        elif length > ctx / lo:
            want = w / factor
            kinds.add("drawn")
        else:
            mix = (ctx / length - lo) / (hi - lo)
            want = (1 - mix) * w / factor + mix * w
            kinds.add("between")
        assert abs(f[i].item() - want) <= 1e-7 * want
    assert c == 1.0 and len(kinds) == 3


def test_frequencies_on_a_ramp(lib):
    theta, r, ctx, factor = 10000.0, 96, 4096, 16.0
    f, c = rope_frequencies(r, theta, "ramp", factor=factor, original_context=ctx)
    at = lambda turns: r * math.log(ctx / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    assert 0 < lo < hi < r // 2
    for i in range(r // 2):
        w = theta ** (-2 * i / r)
        d = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        want = w * (1 - d) + w / factor * d
        assert abs(f[i].item() - want) <= 1e-7 * want
    assert abs(c - (0.1 * math.log(factor) + 1)) < 1e-6


def test_frequencies_per_pair(lib):
    pf = [1.0 + 0.5 * i for i in range(24)]
    f, c = rope_frequencies(48, 10000.0, "per_pair", pair_factors=pf, attn_scale=1.19)
    assert np.allclose(f.numpy(), 10000.0 ** (-np.arange(0, 48, 2) / 48) / np.array(pf), rtol=2e-7) and abs(c - 1.19) < 1e-7


@pytest.mark.parametrize("a,kw", [((0, 1e4), {}), ((63, 1e4), {}), ((64, 1.0), {}), ((64, math.inf), {}), ((64, 1e4, "linear"), dict(factor=0.0)), ((64, 1e4, "linear"), dict(factor=-2.0)),
                                  ((64, 1e4, "by_parts"), dict(factor=8.0)), ((64, 1e4, "by_parts"), dict(factor=8.0, original_context=8192, low_freq=4.0, high_freq=4.0)),
                                  ((64, 1e4, "ramp"), dict(factor=8.0)), ((64, 1e4, "ramp"), dict(factor=8.0, original_context=99, beta_fast=1.0)), ((64, 1e4, "per_pair"), {}),
                                  ((4, 1e4, "per_pair"), dict(pair_factors=[1.0, 0.0])), ((64, 1e4), dict(attn_scale=-1.0)), ((64, 1e4), dict(attn_scale=math.nan))])
def test_frequencies_refusals(lib, a, kw):
    with pytest.raises(RiverError):
        rope_frequencies(*a, **kw)


def test_packed_structs_are_the_headers():
    assert cache_ops._PAGED.size == C.sizeof(cache_ops.river_paged) and cache_ops._ROWS.size == C.sizeof(cache_ops.river_rows)
    b = cache_ops._PAGED.pack(11, 12, 13, *range(1, 9))
    s = cache_ops.river_paged.from_buffer_copy(b)
    assert [getattr(s, n) for n, _ in s._fields_] == [11, 12, 13] + list(range(1, 9))
    r = cache_ops.river_rows.from_buffer_copy(cache_ops._ROWS.pack(5, -6, 1 << 40))
    assert (r.p, r.token, r.head) == (5, -6, 1 << 40)

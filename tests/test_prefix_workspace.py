"""The workspace of attention over shared prefixes: how much a call takes, and how much does for all of them (nothing is launched)."""
import ctypes as C

import pytest

from paper_2604_18396_b200 import prefix_attention_bytes
from tests.test_cache_ops_checks import P, lib, paged  # noqa: F401
from tests.test_prefix_checks import attn

HEADS = ((32, 8, 128), (8, 2, 64), (60, 1, 64), (128, 1, 128), (24, 8, 128))
TOKENS = (0, 1, 2, 63, 64, 65, 500, 1023, 1024, 2047, 2048, 4095, 4096, 4097, 8192, 65536)


def needs(lib, c, n, mq, own, hq):  # noqa: F811
    return lib.river_prefix_attention_needs(C.byref(c), n, mq, own, hq)


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_a_workspace_for_many_does_for_few(hq, hkv, dh):
    for seqs in (1, 2, 16, 64, 300):
        sizes = [prefix_attention_bytes(seqs, n, hq, hkv, dh) for n in TOKENS]
        assert sizes == sorted(sizes) and sizes[0] > 0
        assert all(x <= prefix_attention_bytes(seqs + 1, n, hq, hkv, dh) for x, n in zip(sizes, TOKENS))


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_a_call_takes_what_its_way_needs(lib, hq, hkv, dh):  # noqa: F811
    """At most what does for all, not a byte less than it says; units that are cut (a place of two query tiles' rows, twice for each of 148 CTAs) and, where
    groups have units, two rows for each of the batch's."""
    gq, seen = hq // hkv, set()
    span = 2 * (128 // gq)
    for seqs in (1, 16, 64, 300):
        for n in (1, 16, 64, 300, 500, 2048, 4096, 8192):
            for width in (1, 8, 600, 4096):
                for mq, own in ((1, 1), (1, 100), (1, 0), (n, 100), (n, 0)):
                    c = paged(n_seqs=seqs, max_pages=width, Hkv=hkv, dh=dh)
                    x = needs(lib, c, n, mq, own, hq)
                    assert 0 <= x <= prefix_attention_bytes(seqs, n, hq, hkv, dh)
                    if x == 0:
                        continue
                    cut = 2 * 148 * min(span, n) * gq * (8 + 4 * dh)
                    lists = 148 * 32 + 32 * seqs + 1024
                    rows = [k * n * hq * (8 + 4 * dh) for k in (0, 2)]
                    kind = [k for k in (0, 1) if cut + rows[k] <= x <= cut + rows[k] + lists]
                    assert kind and (0 in kind or n < seqs * span)
                    seen.update(kind)
                    assert attn(lib, c=c, n=n, mq=mq, own=own, hq=hq, q=(P, hq * dh, dh), size=x - 1) == -3
                    assert attn(lib, c=c, n=n, mq=mq, own=own, hq=hq, q=(P, hq * dh, dh), work=0) == -3
    assert seen == {0, 1}


def test_calls_that_need_none(lib):  # noqa: F811
    for kw in (dict(n=0), dict(mq=0), dict(n=-1), dict(mq=-1), dict(own=-1), dict(hq=3), dict(hq=258), dict(n=1 << 29)):
        a = {"n": 64, "mq": 1, "own": 100, "hq": 8, **kw}
        assert needs(lib, paged(n_seqs=64, max_pages=4096), a["n"], a["mq"], a["own"], a["hq"]) == 0, kw
    assert needs(lib, paged(n_seqs=64, max_pages=4096), 64, 1, 100, 8) == prefix_attention_bytes(64, 64, 8, 2, 64)
    assert needs(lib, paged(n_seqs=64, max_pages=4096, dh=96), 64, 1, 100, 8) == 0 and lib.river_prefix_attention_needs(None, 64, 1, 100, 8) == 0

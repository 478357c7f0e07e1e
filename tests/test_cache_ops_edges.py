"""Calls of the operators on a paged cache at their ends, as far as the host alone decides (no GPU)."""
import pytest

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

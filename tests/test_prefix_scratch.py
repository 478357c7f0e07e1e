"""Where who joins parts looks in the scratch (csrc/prefix_plan.h, compiled for the host): within it, whatever a group's note holds."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "prefix_plan.h"
using namespace river;
// A group's note as it stands in the scratch, and a token that looks for its parts there: 0 if the note is not taken, 1 if every row that is read is one of
// n_rows, and of the part's CTA's place or the KV head's rows; else 2.
extern "C" int look(int n_tokens, int Hkv, int gq, long long all, long long share, long long at, int tok0, int n, int keys, int token, int kvh, long long n_rows) {
    const int span = 2 * pf_per(gq);
    const PfPlan p{n_tokens, Hkv * gq, gq, 1, 0, pf_slot_rows(n_tokens, gq)};
    if (!pf_group_has(p, tok0, n, keys, token) || at < 0 || at >= all) return 0;
    const PfUnit u = pf_unit(pf_group_entry(tok0, n, 0, keys, span), (token - tok0) / span, span);
    if (token < u.tok || token >= u.tok + u.n) return 2;
    const int64_t x = kvh * all + at + u.at;
    for (int c = 0; c < kPfCtas; ++c) {
        if (c * share >= x + u.w) break;
        const PfPart r = pf_part(p, share, x, u, c, kvh, 1);
        if (r.k1 <= r.k0) continue;
        const int64_t cut = pf_cut_rows(p), end = r.row + (int64_t)u.n * gq;
        if (r.row < 0 || end > n_rows) return 2;
        if (r.row < cut ? (r.row % p.slot_rows || u.n * gq > p.slot_rows) : end > cut + (int64_t)(kvh + 1) * n_tokens * gq) return 2;
    }
    return 1;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("scratch")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-fwrapv", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2604_18396_b200", "csrc"), str(d / "shim.cpp"), "-o", str(d / "shim.so")])
    return ctypes.CDLL(str(d / "shim.so"))


@pytest.mark.parametrize("seed", range(20))
def test_notes_of_another_call(plan, seed):
    """Starts that descend: no CTA notes the group that a sequence names, and the note of an earlier, larger batch, or anything else, stands in its place."""
    rng = random.Random(seed)
    ll, seen = ctypes.c_longlong, [0, 0]
    for _ in range(3000):
        n_tokens, hkv, gq = rng.choice([1, 3, 40, 700]), rng.choice([1, 2, 8]), rng.choice([1, 3, 4, 12, 60, 128])
        all_ = rng.choice([801, 5000, 10 ** 6, 10 ** 9])
        share = max(640, -(-all_ * hkv // 148))
        some = lambda: rng.choice([0, 1, rng.randint(0, 1000), rng.randint(-2 ** 31, 2 ** 31 - 1), 2 ** 31 - 1])  # noqa: E731
        rows = 2 * 148 * min(2 * (128 // gq), n_tokens) * gq + n_tokens * hkv * gq
        rc = plan.look(n_tokens, hkv, gq, ll(all_), ll(share), ll(rng.choice([0, some(), rng.randint(-2 ** 63, 2 ** 63 - 1)])), some(), some(), some(), rng.randrange(n_tokens),
                       rng.randrange(hkv), ll(rows))
        assert rc in (0, 1)
        seen[rc] += 1
    assert seen[0] and seen[1]

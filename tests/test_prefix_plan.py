"""How attention over shared prefixes is cut into equal parts (csrc/prefix_plan.h), compiled for the host: every key tile of every unit is one
CTA's, and no two parts have a row of the scratch in common."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include <vector>
#include "prefix_plan.h"
using namespace river;
// kinds[i]: 1 group, 0 sequence; returns the number of the first thing that is wrong.  used[row]: how many parts have the row
extern "C" int check(int ctas, int n_tokens, int Hkv, int gq, int groups, int own, int n, const int *kinds, const int *tok0, const int *rows, const int *keys,
                     const int *base, long long n_rows, unsigned char *used, int *most) {
    const int span = 2 * pf_per(gq);
    const PfPlan p{n_tokens, Hkv * gq, gq, groups, own, pf_slot_rows(n_tokens, gq)};
    std::vector<PfEntry> e(n);
    std::vector<int64_t> at(n);
    int64_t all = 0, units = 0;
    for (int i = 0; i < n; ++i) {
        e[i] = kinds[i] ? pf_group_entry(tok0[i], rows[i], 0, keys[i], span) : pf_own_entry(tok0[i], rows[i], 0, base[i], keys[i], span);
        at[i] = all;
        all += e[i].w;
        units += (e[i].n + span - 1) / span;
    }
    const int64_t everything = all * Hkv, share = pf_share(everything, Hkv, units, ctas, own);
    if (share * kPfCtas < everything) return 1;
    *most = 0;
    for (int kvh = 0; kvh < Hkv; ++kvh)
        for (int i = 0; i < n; ++i) {
            const int T = (e[i].n + span - 1) / span;
            int64_t y = 0;
            int seen = 0;
            for (int t = 0; t < T; ++t) {
                const PfUnit u = pf_unit(e[i], t, span);
                if (u.at != y || u.w < kPfCost || pf_unit_at(e[i], y, span) != t || pf_unit_at(e[i], y + u.w - 1, span) != t) return 2;
                if (u.tok != e[i].tok0 + seen || u.n < 1 || u.n > span) return 3;
                if (!kinds[i] && u.keys != pf_max(0, e[i].pos0 + t * span + u.n - e[i].base)) return 4;
                if ((int64_t)u.tiles * kPfKeys < u.keys) return 5;
                const int64_t x = kvh * all + at[i] + y;
                const int c0 = (int)(x / share), c1 = (int)((x + u.w - 1) / share);
                if (c1 >= kPfCtas) return 6;
                int next = 0, parts = 0, whole = 0;
                for (int c = 0; c < kPfCtas; ++c) {
                    const PfPart r = pf_part(p, share, x, u, c, kvh, kinds[i]);
                    if (r.k1 <= r.k0) { if (r.k1 != r.k0) return 7; continue; }
                    if (c < c0 || c > c1 || r.k0 != next) return 8;
                    next = r.k1;
                    ++parts;
                    whole = r.row < 0;
                    if (r.row < 0 && groups) return 9;
                    for (int64_t k = r.row; r.row >= 0 && k < r.row + (int64_t)u.n * gq; ++k) {
                        if (k >= n_rows) return 10;
                        if (used[k]++) return 11;
                    }
                }
                if (next != u.tiles || (whole && parts != 1)) return 12;
                *most = parts > *most ? parts : *most;
                y += u.w;
                seen += u.n;
            }
            if (y != e[i].w || seen != e[i].n) return 13;
        }
    return 0;
}
extern "C" int split(long long units, long long items, int dh) { return pf_split(units, items, dh); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_18396_b200", "csrc"),
                           str(d / "shim.cpp"), "-o", str(d / "shim.so")])
    return ctypes.CDLL(str(d / "shim.so"))


def run(plan, ctas, hkv, gq, groups, own, seqs):
    """seqs: (new tokens, positions, group, shared) in order."""
    from paper_2604_18396_b200 import prefix_attention_bytes
    starts, at = [], 0
    for n, *_ in seqs:
        starts.append(at)
        at += n
    entries = []
    if groups:
        for g in sorted({s[2] for s in seqs}):
            mine = [i for i, s in enumerate(seqs) if s[2] == g]
            rows, sh = sum(seqs[i][0] for i in mine), seqs[mine[0]][3]
            if rows and sh:
                entries.append((1, starts[mine[0]], rows, sh, 0))
    if own:
        entries += [(0, a, n, length, sh if groups else 0) for a, (n, length, _, sh) in zip(starts, seqs) if n]
    n_rows = 2 * 148 * min(2 * (128 // gq), at) * gq + groups * (1 + own) * at * hkv * gq
    used, most = (ctypes.c_ubyte * n_rows)(), ctypes.c_int()
    col = lambda k: (ctypes.c_int * len(entries))(*[e[k] for e in entries])  # noqa: E731
    rc = plan.check(ctas, at, hkv, gq, groups, own, len(entries), col(0), col(1), col(2), col(3), col(4), ctypes.c_longlong(n_rows), used, ctypes.byref(most))
    assert rc == 0, (rc, ctas, hkv, gq, groups, own, seqs)
    if ctas == 148 and (not (groups and own) or at < len(seqs) * 2 * (128 // gq)):  # what the library asks for has room for them
        assert prefix_attention_bytes(len(seqs), at, hkv * gq, hkv, 64) >= n_rows * (8 + 4 * 64) or (groups and at >= len(seqs) * 2 * (128 // gq))
    return most.value


@pytest.mark.parametrize("seed", range(40))
def test_every_tile_is_one_ctas(plan, seed):
    rng = random.Random(seed)
    hkv, gq = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 3, 4, 7, 8, 12, 60, 128])
    groups, own = rng.choice([(1, 0), (1, 1), (0, 1)])
    seqs = []
    for g in range(rng.randint(1, 6)):
        sh = 16 * rng.choice([0, 1, rng.randint(1, 10), rng.randint(1, 500)])
        for _ in range(rng.randint(1, 5)):
            n = rng.choice([0, 1, 1, 2, rng.randint(1, 40), rng.randint(1, 300 // gq + 1)])
            seqs.append((n, sh + n + rng.choice([0, rng.randint(0, 50), rng.randint(0, 5000)]), g, sh))
    if not any(s[0] for s in seqs):
        seqs.append((1, 1, 99, 0))
    for ctas in (1, 2, 7, 148):
        run(plan, ctas, hkv, gq, groups, own, seqs)


def test_lengths_that_are_too_short_for_their_queries(plan):
    for groups, own in ((0, 1), (1, 1)):
        run(plan, 148, 2, 4, groups, own, [(500, 100, 0, 0), (3, 0, 1, 0), (40, 64, 2, 64), (1, 0, 2, 64)])


def test_one_long_prefix_is_everybodys(plan):
    """64 rows of one group over 32 K positions: every CTA has a share of about the same number of tiles."""
    assert run(plan, 148, 8, 4, 1, 0, [(1, 32800, 0, 32768)] * 64) >= 148 // 8


def test_both_kinds_of_work_have_sms(plan):
    ll = ctypes.c_longlong
    for units in (1, 600, 10 ** 5, 10 ** 7, 10 ** 10, 10 ** 14):
        n = [plan.split(ll(units), ll(items), 128) for items in (1, 100, 10 ** 4, 10 ** 6, 10 ** 9, 10 ** 13)]
        assert all(1 <= x <= 148 for x in n) and n == sorted(n, reverse=True)

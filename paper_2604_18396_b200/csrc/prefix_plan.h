// Attention over shared prefixes: what there is to do, and how it is shared out.  Arithmetic on sizes only, without CUDA types, so that it can be
// checked where there is no GPU.
//
// A unit is up to `span` consecutive tokens - two query tiles of 128 / GQ tokens x the GQ query heads of one KV head - with a range of keys:
//   of a group     all tokens of the group's sequences, which follow one another in q, with the positions [0, shared) of its first sequence;
//                  every row sees every key
//   of a sequence  its tokens with the positions from its own first one (`shared`, a whole number of pages) up to the row's own
// Units stand in a row - KV heads outermost, then the groups, then the sequences - and each weighs as many as it has keys, twice that with two
// query tiles, and kPfCost.  That row is cut into equal parts, one per CTA, whatever the lengths are; the CTA of a part computes, of each unit in it, the key tiles that fall between the
// cuts.  A part of a unit leaves per row its O, not divided yet, its maximum and its sum; who joins them finds the same
// cuts by the same arithmetic, or by what the CTAs noted.
#pragma once
#include <cmath>
#include <cstdint>

#ifdef __CUDACC__
#define PF_FN __host__ __device__ __forceinline__
#else
#define PF_FN inline
#endif

namespace river {

constexpr int kPfCtas = 148;   // one per SM of a B200 (were there fewer, the last CTAs would run behind the first: nothing waits between them)
constexpr int kPfKeys = 128;   // of a tile
constexpr int kPfCost = 800;   // what a unit weighs besides its keys (its start and end: 6 us)
constexpr int kPfLeast = 640;  // of a CTA's part: less is not worth its parts' way through memory

PF_FN int pf_per(int gq) { return 128 / gq; }  // tokens of a query tile
template <class T> PF_FN T pf_min(T a, T b) { return b < a ? b : a; }
template <class T> PF_FN T pf_max(T a, T b) { return b > a ? b : a; }

// y / w of numbers that mostly fit 32 bits
PF_FN uint64_t pf_div(uint64_t y, uint64_t w) { return (y | w) >> 32 ? y / w : (uint32_t)y / (uint32_t)w; }

struct PfPlan {
    int n_tokens, Hq, gq;
    int groups, own;  // which units there are: 1, 0: groups' (the sequences' own keys are single tokens'); 1, 1: both; 0, 1: sequences' from their first position on
    int slot_rows;    // rows of a place for a part of a unit
};
// rows of the scratch: two places per CTA for units that are cut, then the groups' and the sequences' whole ones
PF_FN int64_t pf_cut_rows(const PfPlan &p) { return 2 * (int64_t)kPfCtas * p.slot_rows; }
PF_FN int pf_slot_rows(int n_tokens, int gq) { return pf_min(2 * pf_per(gq), n_tokens) * gq; }

// A number of units with one list of keys, in order of their tokens
struct PfEntry {
    int64_t w;  // of all of them; 0: none
    int tok0, n, seq, base, pos0;  // rows; whose row of the table, from which position on; position of the first token (of a sequence)
    int keys;   // of a group
    int group, f;  // f: weight of a key
};
PF_FN PfEntry pf_group_entry(int tok0, int n, int lead, int keys, int span) {
    const int f = 2 * n > span ? 2 : 1;
    return PfEntry{(int64_t)((n + span - 1) / span) * (f * (int64_t)keys + kPfCost), tok0, n, lead, 0, 0, keys, 1, f};
}
PF_FN PfEntry pf_own_entry(int tok0, int n, int seq, int base, int len, int span) {
    const int64_t before = pf_max(0, len - n - base), T = (n + span - 1) / span, f = 2 * n > span ? 2 : 1;
    return PfEntry{(T - 1) * (f * before + kPfCost) + f * (span * T * (T - 1) / 2 + before + n) + kPfCost, tok0, n, seq, base, len - n, 0, 0, (int)f};
}
// the weight of a sequence's units before unit t (t below their number)
PF_FN int64_t pf_before(const PfEntry &e, int t, int span) {
    return t * (e.f * (int64_t)pf_max(0, e.pos0 - e.base) + kPfCost) + e.f * ((int64_t)span * t * (t + 1) / 2);
}
// Unit t of an entry: the weight before it in the entry, its own, its rows, its keys
struct PfUnit {
    int64_t at, w;
    int tok, n, keys, tiles;
};
PF_FN PfUnit pf_unit(const PfEntry &e, int t, int span) {
    PfUnit u;
    u.tok = e.tok0 + t * span;
    u.n = pf_min(span, e.n - t * span);
    if (e.group) {
        u.w = e.f * (int64_t)e.keys + kPfCost;
        u.at = t * u.w;
        u.keys = e.keys;
    } else {
        u.w = e.f * (pf_max(0, e.pos0 - e.base) + (int64_t)t * span + u.n) + kPfCost;
        u.at = pf_before(e, t, span);
        u.keys = pf_max(0, e.pos0 + t * span + u.n - e.base);
    }
    u.tiles = pf_max(1, (u.keys + kPfKeys - 1) / kPfKeys);
    return u;
}
// which unit of an entry stands at weight y
PF_FN int pf_unit_at(const PfEntry &e, int64_t y, int span) {
    if (e.group) return (int)pf_div(y, e.f * (int64_t)e.keys + kPfCost);
    int lo = 0, hi = (e.n + span - 1) / span;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pf_before(e, mid, span) <= y) lo = mid; else hi = mid;
    }
    return lo;
}
// Weight of a CTA's part of `everything`, of about `ctas` CTAs.  Where units are long, of groups that is, as many to each unit, or to each KV head, if that is
// near: parts that begin with a unit spare the CTAs in between a second start and end.
PF_FN int64_t pf_share(int64_t everything, int Hkv, int64_t units, int ctas, int own) {
    auto align = [&](int64_t n) {
        const int64_t to = n > kPfCtas ? 0 : pf_min((ctas + n / 2) / n, kPfCtas / n) * n;
        const bool near = to > 0 && 6 * (to > ctas ? to - ctas : ctas - to) <= ctas;
        if (near) ctas = (int)to;
        return near;
    };
    if (!own && !align(Hkv * pf_max((int64_t)1, units))) align(Hkv);
    return pf_max((int64_t)pf_div(everything + ctas - 1, ctas), (int64_t)kPfLeast);
}
// The tile of a unit that a cut at weight y goes before.  No cut within kPfSnap of a unit's ends, three and a half tiles of one stream: a part of a tile or two would
// cost a CTA more, for its start and end, than another one's share grows.  (us, 0 / 192 / 448 / 896: ragged prompts 79.7 / 79.5 / 79.5 / 77.8, 40 groups of five
// 89.1 / 89.0 / 88.7 / 92.6, 256 rows behind four documents 146.6 / 146.8 / 146.7 / 144.6.)
constexpr int kPfSnap = 448;
PF_FN int pf_cut(int64_t y, int64_t w, int tiles) { return y <= kPfSnap ? 0 : y >= w - kPfSnap ? tiles : (int)pf_div((uint64_t)y * (uint32_t)tiles, (uint64_t)w); }
// What CTA c has of the unit that begins at weight x: tiles k0 .. k1 - 1; its first row among the scratch's (-1: it has all of the unit and the
// rows have nothing else).
struct PfPart {
    int k0, k1;
    int64_t row;
};
PF_FN PfPart pf_part(const PfPlan &p, int64_t share, int64_t x, const PfUnit &u, int c, int kvh, int group) {
    PfPart r;
    const int64_t from = c * share - x;
    r.k0 = pf_cut(from, u.w, u.tiles);
    r.k1 = pf_cut(from + share, u.w, u.tiles);
    if (r.k0 == 0 && r.k1 == u.tiles)
        r.row = p.groups ? pf_cut_rows(p) + (group ? 0 : (int64_t)p.n_tokens * p.Hq) + ((int64_t)kvh * p.n_tokens + u.tok) * p.gq : -1;
    else
        r.row = (2 * (int64_t)c + (from <= 0)) * p.slot_rows;  // (a part that the unit begins in is the CTA's last, another one its first)
    return r;
}

// Whether a group of n tokens from tok0 on, as it was noted at its first sequence, can have the row `token`: then its unit's rows, and the places of their parts
// in the scratch, lie within the batch's.  (Where starts descend, no CTA may have noted the group that a sequence names, and what the scratch held before
// stands there.  INT32_MAX / 2: no row of a table holds more positions.)
PF_FN bool pf_group_has(const PfPlan &p, int tok0, int n, int keys, int token) {
    return tok0 >= 0 && tok0 <= token && token < p.n_tokens && n > token - tok0 && n <= p.n_tokens - tok0 && keys > 0 && keys <= INT32_MAX / 2;
}

// SMs for the groups' units where single tokens run beside them.  u: what the units take, 16 ms for a million of weight with HBM shared; b: what single tokens
// take for `blocks` (K and V of 16 positions of one KV head, 64 dh bytes, at 53 KB/us and SM).  u / x = 10 + b / (n - x): units first, since single tokens
// take the SMs that they leave.  (us, 8B-class heads, with x as said: 64 rows behind 8200 positions 48, x 24 less or more 54, 52; 256 rows behind 9000 to
// 16400 165, 16 less 185, 40 more 170.)
PF_FN int pf_split(int64_t units, int64_t blocks, int dh) {
    const float n = kPfCtas, d = -10.f, u = 16e-3f * (float)units, b = 1.2e-3f * (float)dh * (float)blocks;
    // d x^2 - (d n - u - b) x - u n = 0
    const float p = d * n - u - b, x = -2.f * u * n / (p - sqrtf(p * p + 4.f * d * u * n));
    return pf_min(kPfCtas, pf_max(1, (int)x));
}

}  // namespace river

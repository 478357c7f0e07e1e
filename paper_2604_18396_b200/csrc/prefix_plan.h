// Attention over shared prefixes: what there is to do, and how it is shared out.  Arithmetic on sizes only, without CUDA types, so that it can be
// checked where there is no GPU.
//
// A unit is up to `span` consecutive tokens - two query tiles of 128 / GQ tokens x the GQ query heads of one KV head - with a range of keys:
//   of a group     all tokens of the group's sequences, which follow one another in q, with the positions [0, shared) of its first sequence;
//                  every row sees every key
//   of a sequence  its tokens with the positions from its own first one (`shared`, a whole number of pages) up to the row's own
// Units stand in a row - KV heads outermost, then the groups, then the sequences - and each weighs as many as it has keys, and kPfCost.  That
// row is cut into equal parts, one per CTA, whatever the lengths are; the CTA of a part computes, of each unit in it, the key tiles that fall between the
// cuts.  A part of a unit leaves per row its O, not divided yet, its maximum and its sum; who joins them finds the same cuts by the same arithmetic.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define PF_FN __host__ __device__ __forceinline__
#else
#define PF_FN inline
#endif

namespace river {

constexpr int kPfKeys = 128;   // of a tile
constexpr int kPfCost = 256;   // what a unit weighs besides its keys (its start and end)
constexpr int kPfLeast = 640;  // of a CTA's part: less is not worth its parts' way through memory

PF_FN int pf_per(int gq) { return 128 / gq; }  // tokens of a query tile
template <class T> PF_FN T pf_min(T a, T b) { return b < a ? b : a; }
template <class T> PF_FN T pf_max(T a, T b) { return b > a ? b : a; }

struct PfPlan {
    int ctas, n_tokens, Hq, gq;
    int groups, own;  // which units there are: 1, 0: groups' (the sequences' rows are a step kernel's); 1, 1: both; 0, 1: sequences' from their first position on
    int slot_rows;    // rows of a place for a part of a unit
};
// rows of the scratch: two places per CTA for units that are cut, then the groups' and the sequences' whole ones
PF_FN int64_t pf_cut_rows(const PfPlan &p) { return 2 * (int64_t)p.ctas * p.slot_rows; }
PF_FN int pf_slot_rows(int n_tokens, int gq) { return pf_min(2 * pf_per(gq), n_tokens) * gq; }

// A number of units with one list of keys, in order of their tokens
struct PfEntry {
    int64_t w;  // of all of them; 0: none
    int tok0, n, seq, base, pos0;  // rows; whose row of the table, from which position on; position of the first token (of a sequence)
    int keys;   // of a group
    int group;
};
PF_FN PfEntry pf_group_entry(int tok0, int n, int lead, int keys, int span) {
    return PfEntry{(int64_t)((n + span - 1) / span) * (keys + kPfCost), tok0, n, lead, 0, 0, keys, 1};
}
PF_FN PfEntry pf_own_entry(int tok0, int n, int seq, int base, int len, int span) {
    const int64_t before = pf_max(0, len - n - base), T = (n + span - 1) / span;
    return PfEntry{(T - 1) * (before + kPfCost) + span * T * (T - 1) / 2 + before + n + kPfCost, tok0, n, seq, base, len - n, 0, 0};
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
        u.w = e.keys + kPfCost;
        u.at = t * u.w;
        u.keys = e.keys;
    } else {
        const int64_t before = pf_max(0, e.pos0 - e.base);
        u.at = t * (before + kPfCost) + (int64_t)span * t * (t + 1) / 2;
        u.w = before + t * span + u.n + kPfCost;
        u.keys = pf_max(0, e.pos0 + t * span + u.n - e.base);
    }
    u.tiles = pf_max(1, (u.keys + kPfKeys - 1) / kPfKeys);
    return u;
}
// which unit of an entry stands at weight y
PF_FN int pf_unit_at(const PfEntry &e, int64_t y, int span) {
    if (e.group) return (int)(y / (e.keys + kPfCost));
    const int64_t before = pf_max(0, e.pos0 - e.base);
    int lo = 0, hi = (e.n + span - 1) / span;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (mid * (before + kPfCost) + (int64_t)span * mid * (mid + 1) / 2 <= y) lo = mid; else hi = mid;
    }
    return lo;
}
// weight of a CTA's part of `everything`
PF_FN int64_t pf_share(int64_t everything, int ctas) { return pf_max((everything + ctas - 1) / ctas, (int64_t)kPfLeast); }
// the tile of a unit that a cut at weight y goes before
PF_FN int pf_cut(int64_t y, int64_t w, int tiles) { return y <= 0 ? 0 : y >= w ? tiles : (int)((uint64_t)y * (uint32_t)tiles / (uint64_t)w); }
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

}  // namespace river

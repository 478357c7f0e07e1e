// river_prefix_attention: causal attention over a paged cache whose sequences share prefixes, every shared key read once for its group.
#include <algorithm>
#include <cmath>

#include "prefix_attn_own.cuh"
#include "prefix_attn_tiles.cuh"
#include "tensor_maps.h"

namespace river {
namespace {

enum PrefixMode {
    kPfStep,    // single tokens by themselves: what is shared is read once per sequence
    kPfGroups,  // the groups' keys in query tiles, beside them single tokens with their own keys
    kPfBoth,    // the groups' and the sequences' keys in query tiles, joined row by row
    kPfWhole    // the sequences' rows in query tiles over all of their keys
};
// CTAs of a cluster of single tokens, by an estimate of the time in us: a round of CTAs takes what memory needs for its blocks at `rate` bytes per us, or 0.5
// for each block that a warp has one after the other, and 4 + s / 4 for its start and the joining.  Clusters of more than four leave places free: a GPC,
// of about 16 SMs, takes whole ones.
int own_splits(const PrefixArgs &a, int64_t positions, double rate, double &best_t) {
    const int per_sm = a.c.dh == 128 ? kPfOwnCtas<128> : kPfOwnCtas<64>;
    const double tiles = a.c.Hkv * ((a.p.gq + 7) / 8), units = a.p.n_tokens * tiles, blocks = positions / 16 + 1.0, block_us = 64.0 * a.c.dh / rate;
    const double places_of_queries = (double)a.c.n_seqs * a.max_q * tiles, idle = std::max(0.0, places_of_queries - units) * 0.0015;  // (a CTA leaves where there is no query)
    int best = 1;
    best_t = 1e300;
    for (int s = 1; s <= kStepMaxSplits && places_of_queries * s <= INT32_MAX; ++s) {
        const double places = s <= 4 ? kPfCtas * per_sm : kPfCtas / 18 * (16 * per_sm / s) * s;
        const double turns = 0.5 * std::ceil(blocks / (s * kStepWarps)), stream = places * blocks / s * block_us, fixed = 4.0 + 0.25 * s;
        const double rounds = units * s / places, full = std::floor(rounds), rest = rounds - full;
        const double t = full * (std::max(stream, turns) + fixed) + (rest > 0 ? std::max(stream * rest, turns) + fixed : 0.0) + idle * s;
        if (t < 0.99 * best_t) { best_t = t; best = s; }
    }
    return best;
}
struct PrefixShape {
    PrefixMode mode;
    int splits;  // of single tokens
};

// whether a sequence has fewer rows than a unit has room for, on average: only then do groups' units save keys
bool prefix_both(int n_seqs, int n_tokens, int gq) { return n_tokens < (int64_t)n_seqs * 2 * pf_per(gq); }

// What a call costs in us by each way, and the one that costs least.  `cap`: positions that a row of the table holds, `own`: the most that are a
// sequence's own, as the caller says; how many groups there are the host does not know: one is assumed, and that it has the rest of the row.
//   single tokens     what is shared comes out of L2, at 13 TB/s, but once
//   query tiles       a CTA takes 0.9 us for each of its tiles of up to 128 rows, 1.8 for two of them, and 4 to 8 for a unit's start and end
//   beside them       SMs' shares of HBM (pf_split); 30 us until everything is under way and joined
// (us behind cold caches, single tokens / groups / both / whole; 8B-class heads: 64 rows behind 8200 positions, 20 to 600 of their own 197 / 50 / 72 / 360; 200
// rows in groups of five, 24 query heads, 100 to 2100 shared, f16 97 / 97 / 190 / 266; four beams behind 1500 of the 1B class 12 / 28 / 29 / 25; 108 sequences of
// 6 to 37 tokens in six groups behind up to 332, two heads 190 / 208 / 64 / 36; questions of 17 to 333 tokens in groups of four behind 700 to 2300
// 860 / - / - / 86.)
PrefixShape prefix_shape(const PrefixArgs &a, int max_own) {
    const int gq = a.p.gq, span = 2 * pf_per(gq);
    const int64_t cap = (int64_t)a.c.max_pages << a.c.ps_log2;
    const int own = (int)(max_own ? std::min<int64_t>(max_own, cap) : cap);
    const double heads = a.c.Hkv, rt = (gq + 7) / 8, tokens = a.p.n_tokens, position = 4.0 * a.c.dh * heads;  // (bytes)
    double step_us, own_us;
    const int step = own_splits(a, cap, 13e6, step_us), own_step = own_splits(a, own, 6e6, own_us);
    const double floor_us = ((double)(cap - own) + (double)a.c.n_seqs * own) * position / 6e6;  // (out of HBM)
    step_us = std::max(step_us, 6.0 + floor_us);
    const double rows = tokens * gq, shared_us = heads * std::ceil(rows / 256.0) * ((cap - own) / 128.0 * (rows <= 128 ? 0.9 : 1.8) + 4.0) / kPfCtas;
    const double idle_us = own_us > 1e299 ? 1e300 : std::max(0.0, (double)a.c.n_seqs * a.max_q - tokens) * heads * rt * 0.0015 * own_step;
    own_us = tokens * heads * rt * (own / 16.0 + 6.0) * a.c.dh * 1.2e-3 / kPfCtas + idle_us;
    const double per_seq = std::max(1.0, tokens / a.c.n_seqs), units = heads * a.c.n_seqs * std::ceil(per_seq / span), tile_us = per_seq * gq <= 128 ? 0.9 : 1.8;
    const double own_tiles_us = units * (own / 128.0 * tile_us + 8.0) / kPfCtas, whole_us = std::max(units * (cap / 128.0 * tile_us + 5.0) / kPfCtas, floor_us);
    PrefixShape s = {kPfStep, step};
    double best = step_us;
    const double join_us = std::max(0.0, tokens * heads * rt * (a.c.dh / 32) / (8 * 4 * kPfCtas) - 1.0) * 6.0;  // (rounds behind the first, which 25 and 30 have)
    if (prefix_both(a.c.n_seqs, a.p.n_tokens, gq)) {
        if (30.0 + shared_us + own_us + join_us < best) best = 30.0 + shared_us + own_us + join_us, s = {kPfGroups, own_step};
        if (25.0 + shared_us + own_tiles_us + join_us < best) best = 25.0 + shared_us + own_tiles_us + join_us, s = {kPfBoth, 1};
    }
    if (20.0 + whole_us < best) s = {kPfWhole, 1};
    return s;
}

// The scratch of a call by one way: head, cut units, groups, weights before the sequences, then maxima and sums, and O: of the parts of units that are cut, of the
// groups' whole ones, and of the sequences' whole ones or single tokens' own keys.
struct PrefixScratch {
    size_t cut, group, own_at, ml, o, bytes;
    int64_t own_row;  // the first row of the last kind
};
PrefixScratch prefix_scratch(PrefixMode mode, int n_seqs, int n_tokens, int Hq, int gq, int dh) {
    const int64_t whole = mode == kPfWhole ? 0 : (int64_t)n_tokens * Hq;
    auto behind = [](size_t at, size_t bytes) { return (at + bytes + 127) & ~(size_t)127; };
    PrefixScratch s = {};
    if (mode == kPfStep) return s;
    s.own_row = pf_cut_rows(PfPlan{n_tokens, Hq, gq, 0, 0, pf_slot_rows(n_tokens, gq)}) + whole;
    s.cut = behind(0, sizeof(PfHead));
    s.group = behind(s.cut, kPfCtas * sizeof(PfCut));
    s.own_at = behind(s.group, (size_t)n_seqs * sizeof(PfGroup));
    s.ml = behind(s.own_at, (size_t)n_seqs * sizeof(int64_t));
    s.o = behind(s.ml, (size_t)(s.own_row + whole) * sizeof(float2));
    s.bytes = s.o + (size_t)(s.own_row + whole) * dh * sizeof(float);
    return s;
}
// what every call of up to n_seqs sequences and n_tokens tokens can do with, whichever way it goes
size_t prefix_bytes(int n_seqs, int n_tokens, int Hq, int gq, int dh) {
    const int both = (int)std::min<int64_t>(n_tokens, (int64_t)n_seqs * 2 * pf_per(gq) - 1);  // the most tokens for which groups' units come into question
    return std::max(prefix_scratch(kPfBoth, n_seqs, both, Hq, gq, dh).bytes, prefix_scratch(kPfWhole, n_seqs, n_tokens, Hq, gq, dh).bytes);
}

// a kernel that may start beside the one before it
template <class... P, class... A>
int launch_beside(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, bool beside, A... args) {
    if (smem && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem))) return RIVER_E_DEVICE;
    if (cluster > 8 && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return RIVER_E_DEVICE;
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    if (cluster > 1) {
        at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[cfg.numAttrs++].val.clusterDim = {(unsigned)cluster, 1, 1};
    }
    if (beside) {
        at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    return cuda_rc(cudaLaunchKernelEx(&cfg, kernel, args...));
}
template <class T, int DH>
int launch_tiles(const PrefixArgs &a, const CUtensorMap &map, cudaStream_t st) {
    const size_t smem = prefix_tiles_smem();
    if (cuda_rc(cudaFuncSetAttribute(prefix_tiles_kernel<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem))) return RIVER_E_DEVICE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)kPfCtas);
    cfg.blockDim = dim3(kWpThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cuda_rc(cudaLaunchKernelEx(&cfg, prefix_tiles_kernel<T, DH>, map, a));
}
template <class T, int DH>
int launch(PrefixArgs a, PrefixShape s, cudaStream_t st) {
    const int64_t tiles = (int64_t)a.c.Hkv * ((a.p.gq + 7) / 8), ctas = s.splits * tiles * a.max_q * a.c.n_seqs;  // (of single tokens)
    if ((s.mode == kPfStep || s.mode == kPfGroups) && ctas > INT32_MAX) return RIVER_E_SHAPE;
    a.p.groups = s.mode == kPfGroups || s.mode == kPfBoth;
    a.p.own = s.mode == kPfBoth || s.mode == kPfWhole;
    // the pages of this block, as rows of a head's dims
    CUtensorMap map;
    const size_t rows = (size_t)a.c.n_pages * 2 * a.c.Hkv << a.c.ps_log2;
    if (rows >= (1ull << 31)) return RIVER_E_SHAPE;
    if (!make_map_bf16(&map, a.c.pool + rows * DH * 2 * a.layer0, DH, rows, 16)) return RIVER_E_DEVICE;
    if (s.mode != kPfStep)
        if (const int rc = launch_tiles<T, DH>(a, map, st)) return rc;
    if (s.mode == kPfStep || s.mode == kPfGroups) {
        const int rc = launch_beside(prefix_own_kernel<T, DH>, dim3((unsigned)ctas), 32 * kStepWarps, kPfOwnSmem<DH>, st, s.splits, s.mode == kPfGroups, map, a, s.splits);
        if (rc || s.mode == kPfStep) return rc;
    }
    if (s.mode == kPfWhole) return launch_beside(prefix_join_cut_kernel<T, DH>, dim3(kPfCtas - 1, kJoinBlocks), 256, 0, st, 1, true, a);
    const int64_t joins = (a.p.n_tokens * tiles * (DH / 32) + 7) / 8;
    return launch_beside(joins <= 2 * kPfCtas ? prefix_join_kernel<T, DH, 8, 2> : prefix_join_kernel<T, DH, 3, 4>, dim3((unsigned)joins), 256, 0, st, 1, true, a);
}

// The numbers of a call, checked: what the way of computing and the scratch follow from.
int prefix_numbers(const river_paged *c, int n_tokens, int max_q, int max_own, int Hq, PrefixArgs *a) {
    if (n_tokens < 0 || max_q < 0 || max_own < 0 || Hq < 1 || Hq % c->Hkv) return RIVER_E_BADARG;
    const int gq = Hq / c->Hkv;
    if (c->n_seqs > 8192 || Hq > 8192 || gq > kWpRows || (int64_t)c->n_seqs * Hq > (1 << 26) || (int64_t)n_tokens * Hq > (1 << 30)) return RIVER_E_SHAPE;
    a->max_q = std::min(max_q, n_tokens);
    a->p = PfPlan{n_tokens, Hq, gq, 0, 0, pf_slot_rows(n_tokens, gq)};
    return RIVER_OK;
}
// The arguments of a call, checked.  RIVER_OK with a->n_tokens or a->max_q 0: nothing is to be done.
int prefix_args(const river_paged *c, int layer, int n_tokens, int max_q, int max_own, const int32_t *q_start, const int32_t *lead, const int32_t *shared,
                int Hq, const river_rows *q, float softmax_scale, void *out, const void *workspace, int32_t *status, PrefixArgs *a) {
    *a = PrefixArgs{};
    if (const int rc = paged_check(c, true, true, &a->c)) return rc;
    if (layer < 1 || layer > c->n_layers || !q_start || !lead || !shared || !words(q_start, lead, shared, status) || !std::isfinite(softmax_scale)) return RIVER_E_BADARG;
    if (const int rc = prefix_numbers(c, n_tokens, max_q, max_own, Hq, a)) return rc;
    a->layer0 = layer - 1;
    a->q_start = q_start;
    a->lead = lead;
    a->shared = shared;
    a->scale_log2 = softmax_scale * 1.4426950408889634f;
    a->out = out;
    a->status = status;
    a->polls = kWaitLimit;
    a->mute = -1;
    if (n_tokens == 0) return RIVER_OK;  // (rows that are none may have no address)
    if (!q || !q->p || !out || !aligned_to(out, 16)) return RIVER_E_BADARG;
    // heads are read 16 bytes at a time
    if (!aligned_to(q->p, 16) || q->token % 8 || q->head % 8) return RIVER_E_BADARG;
    a->q = q->p;
    a->q_tok = q->token;
    a->q_head = q->head;
    return aligned_to(workspace, 128) ? RIVER_OK : RIVER_E_BADARG;
}
int launch(PrefixArgs a, int dtype, PrefixShape s, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    const PrefixScratch x = prefix_scratch(s.mode, a.c.n_seqs, a.p.n_tokens, a.p.Hq, a.p.gq, a.c.dh);
    if (x.bytes) {
        if (!workspace || workspace_bytes < x.bytes) return RIVER_E_NOMEM;
        uint8_t *const w = static_cast<uint8_t *>(workspace);
        a.head = reinterpret_cast<PfHead *>(w);
        a.cut = reinterpret_cast<PfCut *>(w + x.cut);
        a.group = reinterpret_cast<PfGroup *>(w + x.group);
        a.own_at = reinterpret_cast<int64_t *>(w + x.own_at);
        a.ml = reinterpret_cast<float2 *>(w + x.ml);
        a.o = reinterpret_cast<float *>(w + x.o);
        a.own_ml = a.ml + x.own_row;
        a.own_o = a.o + x.own_row * a.c.dh;
    }
    return dtype == RIVER_BF16 ? (a.c.dh == 64 ? launch<__nv_bfloat16, 64>(a, s, st) : launch<__nv_bfloat16, 128>(a, s, st))
                               : (a.c.dh == 64 ? launch<__half, 64>(a, s, st) : launch<__half, 128>(a, s, st));
}

}  // namespace
}  // namespace river

using namespace river;

extern "C" size_t river_prefix_attention_bytes(int n_seqs, int n_tokens, int Hq, int Hkv, int dh) {
    if (n_seqs < 1 || n_seqs > 8192 || n_tokens < 0 || Hkv < 1 || Hq < 1 || Hq > 8192 || Hq % Hkv || Hq / Hkv > kWpRows || (dh != 64 && dh != 128)) return 0;
    if ((int64_t)n_tokens * Hq > (1 << 30)) return 0;
    return prefix_bytes(n_seqs, n_tokens, Hq, Hq / Hkv, dh);
}

extern "C" size_t river_prefix_attention_needs(const river_paged *c, int n_tokens, int max_q, int max_own, int Hq) {
    PrefixArgs a = {};
    if (paged_check(c, true, true, &a.c) || prefix_numbers(c, n_tokens, max_q, max_own, Hq, &a) || n_tokens == 0 || max_q == 0) return 0;
    return prefix_scratch(prefix_shape(a, max_own).mode, a.c.n_seqs, n_tokens, Hq, a.p.gq, a.c.dh).bytes;
}

extern "C" int river_prefix_attention(const river_paged *c, int layer, int n_tokens, int max_q, int max_own, const int32_t *q_start, const int32_t *lead,
                                      const int32_t *shared, int Hq, const river_rows *q, float softmax_scale, void *out, void *workspace,
                                      size_t workspace_bytes, int32_t *status, void *cuda_stream) {
    PrefixArgs a;
    if (const int rc = prefix_args(c, layer, n_tokens, max_q, max_own, q_start, lead, shared, Hq, q, softmax_scale, out, workspace, status, &a)) return rc;
    if (a.p.n_tokens == 0 || a.max_q == 0) return RIVER_OK;
    return launch(a, c->dtype, prefix_shape(a, max_own), workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int river_selftest_prefix_attention(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, const int32_t *lead,
                                               const int32_t *shared, int Hq, const river_rows *q, float softmax_scale, void *out, void *workspace,
                                               size_t workspace_bytes, int32_t *status, int way, int mute, int poll_limit, void *cuda_stream) {
    PrefixArgs a;
    if (const int rc = prefix_args(c, layer, n_tokens, max_q, 0, q_start, lead, shared, Hq, q, softmax_scale, out, workspace, status, &a)) return rc;
    if (a.p.n_tokens == 0 || a.max_q == 0 || way < kPfStep || way > kPfWhole || poll_limit < 1 || poll_limit > (1 << 20)) return RIVER_E_BADARG;
    if ((way == kPfGroups || way == kPfBoth) && !prefix_both(c->n_seqs, n_tokens, a.p.gq)) return RIVER_E_SHAPE;
    a.polls = (uint32_t)poll_limit;
    a.mute = mute;
    return launch(a, c->dtype, PrefixShape{(PrefixMode)way, way == kPfStep || way == kPfGroups ? 1 + n_tokens % 4 : 1}, workspace, workspace_bytes,
                  static_cast<cudaStream_t>(cuda_stream));
}

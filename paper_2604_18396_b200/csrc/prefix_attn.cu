// river_prefix_attention: causal attention over a paged cache whose sequences share prefixes, every shared key read once for its group.
#include <algorithm>
#include <cmath>

#include "prefix_attn_step.cuh"
#include "prefix_attn_tiles.cuh"
#include "tensor_maps.h"

namespace river {
namespace {

constexpr int kPfCtas = 148;  // one per SM

enum PrefixMode {
    kPfStep,    // single tokens by themselves: what is shared is read once per sequence
    kPfGroups,  // the groups' keys in query tiles, then single tokens with their own keys
    kPfBoth,    // the groups' and the sequences' keys in query tiles, joined row by row
    kPfWhole    // the sequences' rows in query tiles over all of their keys
};
struct PrefixShape {
    PrefixMode mode;
    int splits;  // of single tokens
};

// whether a sequence has fewer rows than a unit has room for, on average: only then do groups' units save keys, and the scratch has room for them
bool prefix_both(int n_seqs, int n_tokens, int gq) { return n_tokens < (int64_t)n_seqs * 2 * pf_per(gq); }

// What a call costs in us by each way, and the one that costs least.  `cap`: positions that a row of the table holds, `own`: the most that are a
// sequence's own, as the caller says; how many groups there are the host does not know: one is assumed.
PrefixShape prefix_shape(const PrefixArgs &a, int own) {
    const int gq = a.p.gq, span = 2 * pf_per(gq);
    const int64_t cap = (int64_t)a.c.max_pages << a.c.ps_log2;
    WindowArgs w = {};
    w.c = a.c;
    w.n_tokens = a.p.n_tokens;
    w.max_q = a.max_q;
    w.Hq = a.p.Hq;
    w.window = (int)cap;
    double step_us, own_us;
    const int step = step_splits(w, kPfCtas, step_us);
    w.window = own;
    const int own_step = step_splits(w, kPfCtas, own_us);
    // query tiles: a CTA takes 0.9 us for each of its tiles of up to 128 rows, 1.7 for two of them, and some 3 for a unit's start and end
    const double rows = (double)a.p.n_tokens * gq, pairs = std::ceil(rows / 256.0), tile_us = rows <= 128 ? 0.9 : 1.7;
    const double shared_us = 8.0 + a.c.Hkv * pairs * ((cap - std::min<int64_t>(own, cap)) / 128.0 * tile_us + 3.0) / kPfCtas;
    const double per_seq = std::max(1.0, (double)a.p.n_tokens / a.c.n_seqs), units = a.c.n_seqs * std::ceil(per_seq / span);
    const double unit_us = per_seq * gq <= 128 ? 0.9 : 1.7;
    const double own_tiles_us = a.c.Hkv * units * (own / 128.0 * unit_us + 3.0) / kPfCtas;
    const double whole_us = 8.0 + a.c.Hkv * units * (cap / 128.0 * unit_us + 3.0) / kPfCtas;
    PrefixShape s = {kPfStep, step};
    double best = step_us;
    if (prefix_both(a.c.n_seqs, a.p.n_tokens, gq)) {
        if (shared_us + own_us < best) best = shared_us + own_us, s = {kPfGroups, own_step};
        if (shared_us + own_tiles_us + 4.0 < best) s = {kPfBoth, 1};
    } else if (whole_us + 3.0 < best) {
        s = {kPfWhole, 1};
    }
    return s;
}

// The scratch: head, groups, weights before the sequences, then maxima and sums, and O, of `rows` rows.
struct PrefixScratch {
    int64_t rows;
    size_t group, own_at, ml, o, bytes;
};
PrefixScratch prefix_scratch(int n_seqs, int n_tokens, int Hq, int gq, int dh) {
    PrefixScratch s;
    s.rows = pf_cut_rows(PfPlan{kPfCtas, n_tokens, Hq, gq, 0, 0, pf_slot_rows(n_tokens, gq)}) + (prefix_both(n_seqs, n_tokens, gq) ? 2 : 0) * (int64_t)n_tokens * Hq;
    s.group = 128;
    s.own_at = s.group + (size_t)n_seqs * sizeof(PfGroup);
    s.ml = (s.own_at + (size_t)n_seqs * sizeof(int64_t) + 127) & ~(size_t)127;
    s.o = (s.ml + (size_t)s.rows * sizeof(float2) + 127) & ~(size_t)127;
    s.bytes = s.o + (size_t)s.rows * dh * sizeof(float);
    return s;
}


// a kernel that may start beside the one before it
template <class... P, class... A>
int launch_beside(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t st, int cluster, bool beside, A... args) {
    if (cluster > 8 && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return RIVER_E_DEVICE;
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
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
int launch_tiles(const PrefixArgs &a, cudaStream_t st) {
    // the pages of this block, as rows of a head's dims
    CUtensorMap map;
    const size_t rows = (size_t)a.c.n_pages * 2 * a.c.Hkv << a.c.ps_log2;
    if (rows >= (1ull << 31)) return RIVER_E_SHAPE;
    if (!make_map_bf16(&map, a.c.pool + rows * DH * 2 * a.layer0, DH, rows, 16)) return RIVER_E_DEVICE;
    const size_t smem = prefix_tiles_smem();
    if (cuda_rc(cudaFuncSetAttribute(prefix_tiles_kernel<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem))) return RIVER_E_DEVICE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.p.ctas);
    cfg.blockDim = dim3(kWpThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cuda_rc(cudaLaunchKernelEx(&cfg, prefix_tiles_kernel<T, DH>, map, a));
}
template <class T, int DH>
int launch(PrefixArgs a, PrefixShape s, cudaStream_t st) {
    a.p.groups = s.mode == kPfGroups || s.mode == kPfBoth;
    a.p.own = s.mode == kPfBoth || s.mode == kPfWhole;
    if (s.mode != kPfStep)
        if (const int rc = launch_tiles<T, DH>(a, st)) return rc;
    if (s.mode == kPfStep || s.mode == kPfGroups) {
        const int64_t ctas = (int64_t)s.splits * a.c.Hkv * ((a.p.gq + 7) / 8) * a.max_q * a.c.n_seqs;
        if (ctas > INT32_MAX) return RIVER_E_SHAPE;
        return launch_beside(prefix_step_kernel<T, DH>, dim3((unsigned)ctas), 32 * kStepWarps, st, s.splits, s.mode == kPfGroups, a, s.splits);
    }
    if (s.mode == kPfBoth)
        return launch_beside(prefix_join_kernel<T, DH>, dim3((unsigned)std::min<int64_t>(kPfCtas * 8, ((int64_t)a.p.n_tokens * a.p.Hq + 7) / 8)), 256, st, 1, true, a);
    return launch_beside(prefix_join_cut_kernel<T, DH>, dim3(kPfCtas - 1, kJoinBlocks), 256, st, 1, true, a);
}

// The arguments of a call, checked.  RIVER_OK with a->n_tokens or a->max_q 0: nothing is to be done.
int prefix_args(const river_paged *c, int layer, int n_tokens, int max_q, int max_own, const int32_t *q_start, const int32_t *lead, const int32_t *shared,
                int Hq, const river_rows *q, float softmax_scale, void *out, void *workspace, size_t workspace_bytes, int32_t *status, PrefixArgs *a) {
    *a = PrefixArgs{};
    if (const int rc = paged_check(c, true, true, &a->c)) return rc;
    if (layer < 1 || layer > c->n_layers || n_tokens < 0 || max_q < 0 || max_own < 0 || !q_start || !lead || !shared) return RIVER_E_BADARG;
    if (!words(q_start, lead, shared, status) || Hq < 1 || Hq % c->Hkv || !std::isfinite(softmax_scale)) return RIVER_E_BADARG;
    const int gq = Hq / c->Hkv;
    if (c->n_seqs > 65535 || Hq > 8192 || gq > kWpRows || (int64_t)c->n_seqs * Hq > (1 << 26) || (int64_t)n_tokens * Hq > (1 << 30)) return RIVER_E_SHAPE;
    a->layer0 = layer - 1;
    a->max_q = std::min(max_q, n_tokens);
    a->q_start = q_start;
    a->lead = lead;
    a->shared = shared;
    a->scale_log2 = softmax_scale * 1.4426950408889634f;
    a->out = out;
    a->status = status;
    a->p = PfPlan{kPfCtas, n_tokens, Hq, gq, 0, 0, pf_slot_rows(n_tokens, gq)};
    a->polls = kWaitLimit;
    a->mute = -1;
    if (n_tokens == 0) return RIVER_OK;  // (rows that are none may have no address)
    if (!q || !q->p || !out || !aligned_to(out, 16)) return RIVER_E_BADARG;
    // heads are read 16 bytes at a time
    if (!aligned_to(q->p, 16) || q->token % 8 || q->head % 8) return RIVER_E_BADARG;
    a->q = q->p;
    a->q_tok = q->token;
    a->q_head = q->head;
    const PrefixScratch s = prefix_scratch(c->n_seqs, n_tokens, Hq, gq, c->dh);
    if (!workspace || !aligned_to(workspace, 128)) return RIVER_E_BADARG;
    if (workspace_bytes < s.bytes) return RIVER_E_NOMEM;
    uint8_t *const w = static_cast<uint8_t *>(workspace);
    a->head = reinterpret_cast<PfHead *>(w);
    a->group = reinterpret_cast<PfGroup *>(w + s.group);
    a->own_at = reinterpret_cast<int64_t *>(w + s.own_at);
    a->ml = reinterpret_cast<float2 *>(w + s.ml);
    a->o = reinterpret_cast<float *>(w + s.o);
    return RIVER_OK;
}
int launch(const PrefixArgs &a, int dtype, PrefixShape s, cudaStream_t st) {
    return dtype == RIVER_BF16 ? (a.c.dh == 64 ? launch<__nv_bfloat16, 64>(a, s, st) : launch<__nv_bfloat16, 128>(a, s, st))
                               : (a.c.dh == 64 ? launch<__half, 64>(a, s, st) : launch<__half, 128>(a, s, st));
}

}  // namespace
}  // namespace river

using namespace river;

extern "C" size_t river_prefix_attention_bytes(int n_seqs, int n_tokens, int Hq, int Hkv, int dh) {
    if (n_seqs < 1 || n_seqs > 65535 || n_tokens < 0 || Hkv < 1 || Hq < 1 || Hq > 8192 || Hq % Hkv || Hq / Hkv > kWpRows || (dh != 64 && dh != 128)) return 0;
    if ((int64_t)n_tokens * Hq > (1 << 30)) return 0;
    return prefix_scratch(n_seqs, n_tokens, Hq, Hq / Hkv, dh).bytes;
}

extern "C" int river_prefix_attention(const river_paged *c, int layer, int n_tokens, int max_q, int max_own, const int32_t *q_start, const int32_t *lead,
                                      const int32_t *shared, int Hq, const river_rows *q, float softmax_scale, void *out, void *workspace,
                                      size_t workspace_bytes, int32_t *status, void *cuda_stream) {
    PrefixArgs a;
    if (const int rc = prefix_args(c, layer, n_tokens, max_q, max_own, q_start, lead, shared, Hq, q, softmax_scale, out, workspace, workspace_bytes, status, &a)) return rc;
    if (a.p.n_tokens == 0 || a.max_q == 0) return RIVER_OK;
    const int64_t cap = (int64_t)a.c.max_pages << a.c.ps_log2;
    return launch(a, c->dtype, prefix_shape(a, max_own ? (int)std::min<int64_t>(max_own, cap) : (int)cap), static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int river_selftest_prefix_attention(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, const int32_t *lead,
                                               const int32_t *shared, int Hq, const river_rows *q, float softmax_scale, void *out, void *workspace,
                                               size_t workspace_bytes, int32_t *status, int way, int mute, int poll_limit, void *cuda_stream) {
    PrefixArgs a;
    if (const int rc = prefix_args(c, layer, n_tokens, max_q, 0, q_start, lead, shared, Hq, q, softmax_scale, out, workspace, workspace_bytes, status, &a)) return rc;
    if (a.p.n_tokens == 0 || a.max_q == 0 || way < kPfStep || way > kPfWhole || poll_limit < 1 || poll_limit > (1 << 20)) return RIVER_E_BADARG;
    if ((way == kPfGroups || way == kPfBoth) && !prefix_both(c->n_seqs, n_tokens, a.p.gq)) return RIVER_E_SHAPE;
    a.polls = (uint32_t)poll_limit;
    a.mute = mute;
    return launch(a, c->dtype, PrefixShape{(PrefixMode)way, way == kPfStep || way == kPfGroups ? 1 + n_tokens % 4 : 1}, static_cast<cudaStream_t>(cuda_stream));
}

// The units of prefix_plan.h as kernels find them: from a batch's arrays on the device (internal).
#pragma once
#include "prefix_plan.h"
#include "window_attn_rows.cuh"

namespace river {

struct PfHead {
    int64_t all, share;  // weight of one KV head's units; of a CTA's part
};
struct alignas(16) PfCut {  // of a CTA's part: the unit that begins in it and goes on behind it (n 0: none)
    int32_t tok, n, kvh, last;  // its tokens, the CTA that has its last part
    int32_t here, head;         // whether this CTA's rows of it are in the scratch; and those of the unit that began before
};
struct PfGroup {  // at a group's first sequence
    int64_t at;  // the weight before it
    int32_t tok0, n, keys;
};

struct PrefixArgs {
    Paged c;
    PfPlan p;
    int layer0, max_q;
    const int32_t *q_start, *lead, *shared;
    const void *q;
    int64_t q_tok, q_head;
    float scale_log2;
    void *out;
    int32_t *status;
    // scratch
    PfHead *head;
    PfCut *cut;       // [kPfCtas]
    PfGroup *group;   // [n_seqs]
    int64_t *own_at;        // [n_seqs] the weight before a sequence's units
    float2 *ml, *own_ml;    // [rows]: maximum (log2), sum; of units' parts, of single tokens' own keys
    float *o, *own_o;       // [rows][dh]
    uint32_t polls;   // of a wait, before it gives up
    int mute;         // self-test: the KV head whose keys nobody asks for, so that waits run out
};

// positions that a group shares: whole pages that its row of the table can hold
__device__ __forceinline__ int pf_shared(const Paged &c, int v) { return max(0, min(v, c.max_pages << c.ps_log2)) & ~((1 << c.ps_log2) - 1); }
__device__ __forceinline__ int pf_len(const Paged &c, int len) { return max(0, min(len, c.max_pages << c.ps_log2)); }
// whether sequence s goes on with the group of the one before it
__device__ __forceinline__ bool pf_linked(const PrefixArgs &a, int s) { return s > 0 && a.lead[s] != s && a.lead[s] == a.lead[s - 1] && a.shared[s] == a.shared[s - 1]; }
// whether what the batch's arrays say of sequence s is as it should be
__device__ __forceinline__ bool pf_sound(const PrefixArgs &a, int s) {
    const int x = a.q_start[s], y = a.q_start[s + 1], len = a.c.lens[s], sh = a.shared[s];
    return x >= 0 && y >= x && y <= a.p.n_tokens && y - x <= a.max_q && len >= 0 && len <= (a.c.max_pages << a.c.ps_log2) && sh == pf_shared(a.c, sh) && (sh == 0 || len - (y - x) >= sh) &&
           (a.lead[s] == s || pf_linked(a, s));
}
// entries of a KV head: groups, each where its last sequence stands, then sequences
__device__ __forceinline__ int pf_entries(const PrefixArgs &a) { return a.c.n_seqs * (a.p.groups + a.p.own); }
__device__ __forceinline__ PfEntry pf_entry(const PrefixArgs &a, int i, int span) {
    const int S = a.c.n_seqs;
    const bool group = a.p.groups && i < S;
    const int s = a.p.groups && !group ? i - S : i, l = group ? a.lead[s] : s, shared = a.p.groups ? pf_shared(a.c, a.shared[s]) : 0;
    if (group && (shared == 0 || l < 0 || l > s || (s + 1 < S && pf_linked(a, s + 1)))) return PfEntry{};
    const int t0 = a.q_start[l], t1 = a.q_start[s + 1];
    if (t0 < 0 || t1 <= t0 || t1 > a.p.n_tokens) return PfEntry{};
    return group ? pf_group_entry(t0, t1 - t0, l, shared, span) : pf_own_entry(t0, t1 - t0, s, shared, pf_len(a.c, a.c.lens[s]), span);
}

// blocks of 16 positions of one KV head that single tokens of sequence s read
__device__ __forceinline__ int64_t pf_blocks(const PrefixArgs &a, int s) {
    const int n = a.q_start[s + 1] - a.q_start[s], base = pf_shared(a.c, a.shared[s]), len = pf_len(a.c, a.c.lens[s]);
    return n > 0 && n <= a.p.n_tokens ? (int64_t)n * ((max(0, len - base) >> 4) + 6) : 0;
}

// Exclusive prefix sum of x over the 128 threads of warps 0 .. 3, whose sum is added to `total`, and that of y to `other` (part: one per warp).  Ends with a
// barrier of theirs (number 3) behind every read.
__device__ __forceinline__ void pf_scan_sync() { asm volatile("bar.sync 3, 128;" ::: "memory"); }
__device__ __forceinline__ int64_t pf_scan(int64_t x, int64_t y, longlong2 *part, int64_t &total, int64_t &other) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t z = __shfl_up_sync(0xffffffffu, inc, o);
        y += __shfl_xor_sync(0xffffffffu, y, o);
        if (lane >= o) inc += z;
    }
    if (lane == 31) part[warp] = make_longlong2(inc, y);
    pf_scan_sync();
    int64_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const longlong2 z = part[w];
        if (w < warp) before += z.x;
        sum += z.x;
        other += z.y;
    }
    total += sum;
    pf_scan_sync();
    return before + inc - x;
}

}  // namespace river

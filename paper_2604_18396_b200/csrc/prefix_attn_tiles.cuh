// Attention over shared prefixes on tcgen05 (sm_100a, internal): the units of prefix_units.cuh.
//
// One CTA per SM walks its part of the row of units, 128 keys at a time, without a stop between units: the loads of the next one are under way
// while a unit ends.
//   S [128 x 128] = Q K^T     Q and K in shared memory, S in tensor memory
//   O [128 x DH] += P V       P (rounded to the inputs' type) in tensor memory over the place of S, V as it lies in the cache
//   warp 0        TMA: K and V pages, one 16 x 64 box per lane, three places for K, two for V
//   warp 1        tensor memory; one lane issues the MMAs: P V of a stream, S of its next keys, then the other stream's, so that the softmax of
//                 one runs under the MMAs of the other
//   warp 2        the parts of units, one ahead
//   warps 4..11   softmax, four per stream: thread = query row = TMEM lane; online, base 2, fp32; all 128 scores of a row in registers; O is
//                 rescaled only when a row's maximum has grown by more than 2^8 since it last was.  P goes out in two halves.
// Two streams: the two query tiles of a unit, over the same K and V; or, where a unit has one query tile, its even and its odd key tiles, joined
// through shared memory when the keys are through (dual).
//
// P in 16 bits: its rounding weighs as much as the rounding of the result (2^-9 of sum p |v| against 2^-9 of the result in bf16, both
// random).  In f16 a probability below 2^-21 of the row's largest loses bits, and below 2^-31 it counts as 2^-31 (kWpBelow).
//
// Hidden positions: scores are replaced, not added to; V rows that no row of the unit sees are set to zero in shared memory.  A row of V
// that some rows see and others do not is harmless as long as it is finite (0 x v); tiles that have such rows are looked through (f16: all
// of their rows), and where one holds an infinity or no number the part is computed again row by row (pf_row), while the CTA's other warps
// wait for as long as that moves on.  So it is for scores beyond kWpHuge.  (256 rows of 4096 positions: 60 ms.)
//
// Bound by the tensor pipe and the special-function units alike, both two thirds active: 16 prompts of 512 behind 8192 positions, 8B-class heads, 1.13
// TFLOP in 855 us, 1.32 PFLOP/s (a burst; in a loop of seconds 1.12, by the power cap).  A key tile of two query tiles takes 1.65 us, of one 0.9, and 2.3 beside
// single tokens that stream; a unit's start and end 6; until the first scores behind cold caches it is 11 us, 5 of them until the units are found.  Two
// threads per query row, 16 warps of softmax, would have 902 us for those 855; a loop for the MMA warp's places 2.1 us a tile.
#pragma once
#include "prefix_units.cuh"
#include "window_attn_prompt.cuh"

namespace river {

// A part of a unit, as the warps of a CTA hand it on
struct PfSeg {
    int n_kt, t0;          // key tiles (0: that was the last part), the first one
    int tok0, n_tok, kvh;  // rows
    int seq, base, keys;   // whose row of the table, from which position on, how many
    int causal, pos0;      // a sequence's unit: position of the first token
    int64_t row;           // first row in the scratch; -1: the result's
};

// x, of which the compiler knows nothing: a loop is not written twice for what does not change in it (the kernel's code would be three times as long, and
// fetching it behind cold caches is a third of a small call).
__device__ __forceinline__ int opaque(int x) {
    asm volatile("" : "+r"(x));
    return x;
}
// One row over the positions [lo, hi) of a row of the table, by one warp in their order: O (not divided), maximum and sum.  A position takes half a microsecond:
// `moved` goes up every 128 of them, for those who wait.
template <class T, int DH>
__device__ void pf_row(const PrefixArgs &a, int token, int head, int seq, int lo, int hi, float (&o)[DH / 32], float &m, float &l, int *moved) {
    constexpr int E = DH / 32;
    const int lane = threadIdx.x & 31, kvh = head / a.p.gq, pmask = (1 << a.c.ps_log2) - 1;
    const T *q = static_cast<const T *>(a.q) + token * a.q_tok + head * a.q_head + E * lane, *pool = reinterpret_cast<const T *>(a.c.pool);
    float x[E];
    m = -CUDART_INF_F;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) { x[e] = to_f(q[e]) * a.scale_log2; o[e] = 0.f; }
#pragma unroll 1
    for (int j = lo; j < hi; ++j) {
        if (lane == 0 && ((j - lo) & 127) == 0) atomicAdd(moved, 1);
        const int col = j >> a.c.ps_log2, page = col < a.c.max_pages ? a.c.table[(size_t)seq * a.c.max_pages + col] : -1;
        if (page < 0 || page >= a.c.n_pages) continue;
        const T *k = pool + a.c.row(a.layer0, page, 0, kvh, j & pmask) + E * lane, *v = pool + a.c.row(a.layer0, page, 1, kvh, j & pmask) + E * lane;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += x[e] * to_f(k[e]);
        s = warp_sum(s);
        const float mx = fmaxf(m, s), base = mx == -CUDART_INF_F ? 0.f : mx, corr = exp2f(m - base), p = exp2f(s - base);
        m = mx;
        l = l * corr + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * corr + p * to_f(v[e]);
    }
}

// The rows of a part, one by one (warps 4 .. 11)
template <class T, int DH>
__device__ __noinline__ void pf_rows_again(const PrefixArgs &a, const PfSeg &g, int *moved) {
    const int gq = a.p.gq, lane = threadIdx.x & 31;
#pragma unroll 1
    for (int x = (threadIdx.x >> 5) - 4; x < g.n_tok * gq; x += 8) {
        const int token = g.tok0 + x / gq, head = g.kvh * gq + x % gq, lo = g.base + kPfKeys * g.t0;
        const int hi = g.base + min(min(g.keys, kPfKeys * (g.t0 + g.n_kt)), g.causal ? g.pos0 + x / gq + 1 - g.base : g.keys);
        float o[DH / 32], m, l;
        pf_row<T, DH>(a, token, head, g.seq, lo, hi, o, m, l, moved);
        if (g.row >= 0 && lane == 0) a.ml[g.row + x] = make_float2(m, l);
#pragma unroll
        for (int e = 0; e < DH / 32; ++e) {
            const int d = DH / 32 * lane + e;
            if (g.row < 0) static_cast<T *>(a.out)[((size_t)token * a.p.Hq + head) * DH + d] = from_f<T>(l == 0.f ? 0.f : o[e] / l);
            else a.o[g.row * DH + ((int64_t)(d >> 2) * (g.n_tok * gq) + x) * 4 + (d & 3)] = o[e];
        }
    }
}

template <class T, int DH>
__global__ void __launch_bounds__(kWpThreads, 1) prefix_tiles_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ PrefixArgs a) {
    constexpr int NB = DH / 64;                                          // blocks of 64 dims
    constexpr bool kHalf = std::is_same<T, __half>::value;
    constexpr uint32_t QB = kWpRows * 128, KB = kWpKeys * 128;           // bytes of one block of Q / of K or V
    constexpr uint32_t kO = 256;                                         // TMEM: stream q has S / P in columns 128 q .., O in 256 + DH q ..
    constexpr uint32_t kIdS = (1u << 4) | (kHalf ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(kWpRows >> 4) << 24) | ((uint32_t)(kWpKeys >> 3) << 17);
    constexpr uint32_t kIdO = (kIdS & ~(0x3Fu << 17)) | ((uint32_t)(DH >> 3) << 17) | (1u << 16);  // (B of the second product: N-major)
    extern __shared__ uint8_t wp_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(wp_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *const sq = smem, *const sv = sq + 2 * NB * QB, *const sk = sv + 2 * NB * KB;  // [tile], [2 places of V], [3 of K] [NB][128 rows][128 bytes]
    // K of the first tile there; V of tile i and K of tile i + 1 there (4, in turn; tiles are counted over all units); V and K of tile i before
    // free (2); per stream: S done (2), P written (2 x 2), O done (2); Q there; a part there (2), no longer needed (2)
    __shared__ uint64_t bars[20];
    __shared__ longlong2 s_part[4];
    __shared__ int64_t s_at;
    __shared__ PfEntry s_entry;  // the first one that this CTA has units of
    __shared__ PfSeg s_seg[2];
    __shared__ float2 s_ml[kWpRows];  // dual: the second stream's maxima and sums
    __shared__ uint32_t s_tmem;
    __shared__ int s_first, s_kvh, s_abort, s_no_page, s_poison[2], s_missing[2];
    __shared__ int s_moved;  // counted up while rows are computed again, which may take longer than the polls of those who wait for its end
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int gq = a.p.gq, per = pf_per(gq), span = 2 * per, S = a.c.n_seqs, D = pf_entries(a);
    const uint32_t b_first = smem_u32(&bars[0]), b_full = b_first + 8, b_free = b_full + 32, b_s = b_free + 16, b_p = b_s + 16, b_o = b_p + 32, b_q = b_o + 16,
                   b_seg = b_q + 8, b_used = b_seg + 16;
    volatile int *abortp = &s_abort;
    pdl_launch();  // (whatever starts beside this kernel takes no tensor memory)
    if (tid == 0) {
        s_abort = s_moved = s_no_page = s_poison[0] = s_poison[1] = s_missing[0] = s_missing[1] = 0;
        s_first = -1;
#pragma unroll 1
        for (int i = 0; i < 20; ++i) mbar_init(smem_u32(&bars[i]), i >= 9 && i < 13 ? 4 : i == 15 ? 8 : i >= 18 ? 10 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }

    // the queries, on their way to L2 while the parts are found (as far as one line per thread reaches)
    {
        const int64_t x = (int64_t)blockIdx.x * kWpThreads + tid, lines = (int64_t)a.p.Hq * (DH / 64);
        if (x < a.p.n_tokens * lines) {
            const int token = (int)pf_div(x, lines), y = (int)(x - token * lines);
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T *>(a.q) + token * a.q_tok + y / (DH / 64) * a.q_head + y % (DH / 64) * 64));
        }
    }
    if (warp == 1) {
        tc_alloc(smem_u32(&s_tmem), 512u);
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(s_tmem);
    // the next part; whether there is one.  `used`: told at once that it has been read
    auto take = [&](int n, PfSeg &g) {
        wp_wait(b_seg + 8 * (n & 1), n >> 1, &s_moved, abortp, a.polls);
        g = s_seg[n & 1];
        return g.n_kt > 0 && !__any_sync(0xffffffffu, *abortp);
    };
    auto used = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(b_used + 8 * (n & 1));
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ---- this CTA's part of the row of units
        const bool beside = a.p.groups && !a.p.own;  // single tokens run on the other SMs
        PfEntry mine = {};
        int64_t all = 0, blocks = 0, at = 0, none = 0;  // (blocks of single tokens; from bit 44 on, units of a KV head)
#pragma unroll 1
        for (int i0 = 0; i0 < D; i0 += 128) {
            const int i = i0 + tid;
            mine = i < D ? pf_entry(a, i, span) : PfEntry{};
            at = all + pf_scan(mine.w, beside && i < D ? pf_blocks(a, i) + ((int64_t)((mine.n + span - 1) / span) << 44) : 0, s_part, all, blocks);
        }
        const int64_t everything = all * a.c.Hkv, share = pf_share(everything, a.c.Hkv, blocks >> 44, beside ? pf_split(everything, (blocks & ((1ll << 44) - 1)) * a.c.Hkv * ((gq + 7) / 8), a.c.dh) : kPfCtas, a.p.own);
        const int64_t x0 = blockIdx.x * share, x1 = min(x0 + share, everything);
        if (x0 < everything || blockIdx.x == 0) {
            const int kvh0 = all ? (int)pf_div(x0, all) : 0;
            const int64_t xl = x0 - kvh0 * all;
            int64_t base = 0;
#pragma unroll 1
            for (int i0 = 0; i0 < D; i0 += 128) {
                const int i = i0 + tid;
                if (D > 128) {  // (else they are known)
                    mine = i < D ? pf_entry(a, i, span) : PfEntry{};
                    at = base;
                    at += pf_scan(mine.w, 0, s_part, base, none);
                }
                if (mine.w && at <= xl && xl < at + mine.w) s_first = i, s_kvh = kvh0, s_at = at, s_entry = mine;
                if (blockIdx.x == 0 && i < D) {  // for who joins the parts
                    if (!a.p.groups || i >= S) a.own_at[a.p.groups ? i - S : i] = at;
                    else if (mine.w) a.group[mine.seq] = PfGroup{at, mine.tok0, mine.n, mine.keys};
                }
            }
            if (blockIdx.x == 0) {
                if (tid == 0) a.head->all = all, a.head->share = share;
#pragma unroll 1
                for (int s = tid; s < S; s += 128)
                    if (!pf_sound(a, s)) flag(a.status, RIVER_E_BADARG);
            }
        }
        pf_scan_sync();
        if (warp == 2) {  // ---- the parts
            int64_t x = x0, ent = s_at;  // (ent: the weight before the entry, of this KV head)
            int i = s_first, kvh = s_kvh, n = 0;
            if (lane == 0) a.cut[blockIdx.x] = PfCut{};
            PfEntry e = s_entry;
#pragma unroll 1
            while (x < x1) {
                int64_t y = x - kvh * all - ent;  // within the entry
#pragma unroll 1
                for (int t = pf_unit_at(e, y, span); x < x1 && y < e.w; ++t) {
                    const PfUnit u = pf_unit(e, t, span);
                    const PfPart p = pf_part(a.p, share, x - y + u.at, u, blockIdx.x, kvh, e.group);
                    if (p.k1 > p.k0) {
                        if (n >= 2) wp_wait(b_used + 8 * (n & 1), (n >> 1) - 1, &s_moved, abortp, a.polls);
                        if (lane == 0) {
                            s_seg[n & 1] = PfSeg{p.k1 - p.k0, p.k0, u.tok, u.n, kvh, e.seq, e.base, u.keys, !e.group, e.pos0 + u.tok - e.tok0, p.row};
                            mbar_arrive(b_seg + 8 * (n & 1));
                        }
                        ++n;
                    }
                    if (lane == 0) {  // for who joins the parts
                        const int64_t from = x - y + u.at, to = from + u.w;
                        const int there = p.k1 > p.k0 && p.row >= 0;
                        if (from < x0) a.cut[blockIdx.x].head = there;
                        else if (to > x0 + share) *reinterpret_cast<int4 *>(a.cut + blockIdx.x) = make_int4(u.tok, u.n, kvh, (int)pf_div(to - 1, share)), a.cut[blockIdx.x].here = there;
                    }
                    x += u.at + u.w - y;
                    y = u.at + u.w;
                }
                if (x >= x1 || __any_sync(0xffffffffu, *abortp)) break;
                // the next entry that has units: from behind this one, or the next KV head's first
                ent += e.w;
                int i0 = i + 1;
#pragma unroll 1
                while (kvh < a.c.Hkv) {  // (always: there is weight left, unless somebody writes the batch's arrays meanwhile)
                    if (i0 >= D) i0 = 0, ++kvh, ent = 0;
                    const unsigned there = __ballot_sync(0xffffffffu, i0 + lane < D && pf_entry(a, i0 + lane, span).w > 0);
                    if (there) {
                        i = i0 + __ffs(there) - 1;
                        break;
                    }
                    i0 += 32;
                }
                if (kvh >= a.c.Hkv) break;
                e = pf_entry(a, i, span);
            }
            if (n >= 2) wp_wait(b_used + 8 * (n & 1), (n >> 1) - 1, &s_moved, abortp, a.polls);
            if (lane == 0) {
                s_seg[n & 1].n_kt = 0;
                mbar_arrive(b_seg + 8 * (n & 1));
            }
        } else if (warp == 0) {  // ---- K and V
            const int blk = lane / NB, half = lane % NB, bpp = a.c.ps_log2 - 4;
            PfSeg g, f;  // of the tile whose V is loaded, of the one whose K is
            int n = 0, j = -1, place = 0;
            auto page_of = [&](const PfSeg &s, int t) {  // of this lane's block of tile t; -1: none
                const int u = 8 * (s.t0 + t) + blk, col = ((s.base >> 4) + u) >> bpp;
                const int page = blk < 8 && t < s.n_kt && 16 * u < s.keys && col < a.c.max_pages ? a.c.table[(size_t)s.seq * a.c.max_pages + col] : -1;
                return page < a.c.n_pages ? max(page, -1) : -1;
            };
            auto load = [&](const PfSeg &s, int t, uint8_t *dst, int page, int v, uint32_t bar) {
                const int row = ((page * 2 * a.c.Hkv + s.kvh + v * a.c.Hkv) << a.c.ps_log2) + ((s.base + 16 * (8 * (s.t0 + t) + blk)) & ((1 << a.c.ps_log2) - 1));
                if (page >= 0) tma_load_2d(smem_u32(dst) + half * KB + blk * 2048, &tmap, 64 * half, row, bar);
            };
            bool more = take(n, f);
            used(n++);
            if (more && f.kvh == a.mute) more = false;
            int jf = 0, page = -1, ahead = more ? page_of(f, 0) : -1;
            uint32_t bytes = 0;
#pragma unroll 1
            for (int i = -1; more || i >= 0; ++i) {
                // V of tile i (g, j), K of tile i + 1 (f, jf)
                const int next = more ? ahead : -1;
                if (more) {
                    if (blk < 8 && 16 * (8 * (f.t0 + jf) + blk) < f.keys && next < 0) s_no_page = 1;
                    ahead = page_of(f, jf + 1);  // (under way while this tile waits for its place)
                }
                const uint32_t k_bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, next >= 0)) * 2048u, bar = i < 0 ? b_first : b_full + 8 * (i & 3);
                if (i >= 2) wp_wait(b_free + 8 * (i & 1), (i >> 1) - 1, &s_moved, abortp, a.polls);
                if (__any_sync(0xffffffffu, *abortp)) break;
                if (lane == 0) mbar_expect_tx(bar, bytes + k_bytes);
                __syncwarp();
                if (more) load(f, jf, sk + place * NB * KB, next, 0, bar);
                if (i >= 0) load(g, j, sv + (i & 1) * NB * KB, page, 1, bar);
                if (!more) break;
                page = next;
                bytes = k_bytes;
                place = place == 2 ? 0 : place + 1;
                g = f;
                j = jf;
                if (++jf == f.n_kt) {
                    more = take(n, f);
                    used(n++);
                    jf = 0;
                    ahead = more ? page_of(f, 0) : -1;
                }
            }
        } else if (warp == 1) {  // ---- the products
            const uint64_t dq = tc_smem_desc(smem_u32(sq)), dk = tc_smem_desc(smem_u32(sk)), dv = pt_desc_n(smem_u32(sv), KB);
            const bool leader = elect_one();
            PfSeg g;
            int i0 = 0, cp0 = 0, cp1 = 0;  // tiles of the parts before; of each stream
            int k_i = 0, place = 0;        // K of tile k_i is next, at `place`
            auto scores = [&](int q, int tile) {  // S of stream q: query tile `tile` and the next K
                wp_wait(k_i == 0 ? b_first : b_full + 8 * ((k_i - 1) & 3), k_i == 0 ? 0 : (k_i - 1) >> 2, abortp, a.polls);
                tc_fence_after();
                const uint64_t k_desc = dk + place * (NB * KB >> 4);
                if (leader) {
#pragma unroll
                    for (int k = 0; k < DH / 16; ++k)
                        tc_mma(tmem + 128u * q, dq + (tile * NB + (k >> 2)) * (QB >> 4) + 2 * (k & 3), k_desc + (k >> 2) * (KB >> 4) + 2 * (k & 3), kIdS, k ? 1u : 0u);
                    tc_commit(b_s + 8 * q);
                }
                __syncwarp();
            };
            auto next_k = [&] { ++k_i; place = place == 2 ? 0 : place + 1; };
            auto values = [&](int q, int i, int count, bool fresh, bool frees) {  // O of stream q += P V of tile i
                const uint64_t v = dv + (i & 1) * (NB * KB >> 4);
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // half of the keys
                    wp_wait(b_p + 8 * (2 * q + h), count, abortp, a.polls);
                    tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)  // 16 keys: 8 columns of P, 2048 bytes of V
                            tc_mma_ts(tmem + kO + (uint32_t)DH * q, tmem + 128u * q + 32 * h + 8 * k, v + (4 * h + k) * (2048 >> 4), kIdO, !fresh || h || k ? 1u : 0u);
                        if (h == 1 && frees) tc_commit(b_free + 8 * (i & 1));
                    }
                    __syncwarp();
                }
            };
            for (int n = 0;; ++n) {
                const bool more = take(n, g);
                used(n);
                if (!more) break;
                const int n_t = uniform(g.n_kt), nq = g.n_tok > per ? 2 : 1;
                const bool dual = nq == 1 && n_t > 1;
                wp_wait(b_q, n, &s_moved, abortp, a.polls);
                scores(0, 0);
                if (dual) {
                    next_k();
                    scores(1, 0);
                } else if (nq == 2) scores(1, 1);
                next_k();
                for (int j = 0; j < n_t; ++j) {
                    const int i = i0 + j;
                    wp_wait(b_full + 8 * (i & 3), i >> 2, abortp, a.polls);
                    if (dual) {
                        const int q = j & 1;
                        values(q, i, q ? cp1++ : cp0++, j < 2, true);
                        if (j + 2 < n_t) {
                            scores(q, 0);
                            next_k();
                        } else if (leader) tc_commit(b_o + 8 * q);
                    } else {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (q == nq) break;
                            values(q, i, q ? cp1++ : cp0++, j == 0, q == nq - 1);
                            if (j + 1 < n_t) scores(q, q);
                            else if (leader) tc_commit(b_o + 8 * q);
                        }
                        if (j + 1 < n_t) next_k();
                    }
                    __syncwarp();
                    if (*abortp) break;
                }
                i0 += n_t;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int q = (warp - 4) >> 2, r = 32 * (warp & 3) + lane, u0 = tid - 128, inv_gq = 65536 / gq + 1;  // (r * inv_gq >> 16 = r / gq for r < 128)
        const uint32_t turn = a.scale_log2 < 0.f ? 0x80008000u : 0u;
        const uint32_t quarter = (uint32_t)(32 * (warp & 3)) << 16, t_s = tmem + 128u * q + quarter, t_o = tmem + kO + (uint32_t)DH * q + quarter;
        const float c = fmaxf(fabsf(a.scale_log2), 1e-30f);  // (a scale of 0: every score 0, hidden ones -inf still)
        const int bpp = a.c.ps_log2 - 4;
        PfSeg g;
        int i0 = 0, count = 0, ended = 0;  // tiles of the parts before; tiles, and parts, of this stream
        // Part -1 is none: a tile of each stream on whatever tensor memory holds, without waits and arrivals, while this CTA's part of the units is looked for.
        // It fetches the code: a first tile takes 6 us behind cold caches, where the others take 1.7.  Not where single tokens take the SM if this CTA has no part: that
        // the last third of the CTAs has none is likely.  (us, in no CTA / in the first 96 / in all: 64 rows of a group 46.3 / 44.9 / 43.4, 256 rows of four 147.4 /
        // 146.7 / 147.8, 40 groups of five 90.8 / 88.7 / 88.4.)
#pragma unroll 1
        for (int n = a.p.own || blockIdx.x < 96 ? -1 : 0;; ++n) {
            const bool dry = n < 0;
            if (dry) {
                g = PfSeg{2, 0, 0, 0, 0, 0, 0, 2 * kPfKeys, 0, 0, 0};
            } else {
                // the part before: where something in it was no number, its rows again
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (n > 0 && s_poison[(n - 1) & 1] && !*abortp) pf_rows_again<T, DH>(a, g, &s_moved);
                if (n > 0) used(n - 1);
                {  // one answer for all eight warps: nobody leaves while others wait at a barrier
                    const bool more = take(n, g);
                    uint32_t none = more ? 0u : 1u;
                    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %0, 0;\n\tbarrier.cta.red.or.pred p, 1, 256, q;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "+r"(none)::"memory");
                    if (none) break;
                }
                {  // ---- Q rows in the operand's swizzled order (a negative scale turns their signs); rows that are none are zero
                    constexpr int C8 = DH / 8;  // 16-byte chunks of a row; all of a thread's are under way together
                    const int c8 = u0 % C8;
                    const T *src = static_cast<const T *>(a.q) + g.tok0 * a.q_tok + g.kvh * gq * a.q_head + 8 * c8;
                    auto place = [&](int rr) { const int rx = rr % kWpRows; return sq + rr / kWpRows * NB * QB + (c8 >> 3) * QB + rx * 128 + (((c8 & 7) ^ (rx & 7)) * 16); };
    #pragma unroll 4
                    for (int i = 0; i < C8; ++i) {
                        const int rr = u0 / C8 + i * (256 / C8), rx = rr % kWpRows, pp = rx * inv_gq >> 16, p = rr / kWpRows * per + pp, h = rx - pp * gq;
                        const bool on = pp < per && p < g.n_tok;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(place(rr))), "l"(on ? src + p * a.q_tok + h * a.q_head : src), "r"(on ? 16 : 0) : "memory");
                    }
                    bool missing = false;
    #pragma unroll 1
                    for (int u = 8 * g.t0 + u0; u < 8 * (g.t0 + g.n_kt) && 16 * u < g.keys; u += 256) {
                        const int col = ((g.base >> 4) + u) >> bpp, page = col < a.c.max_pages ? a.c.table[(size_t)g.seq * a.c.max_pages + col] : -1;
                        missing = missing || page < 0 || page >= a.c.n_pages;
                    }
                    if (missing) s_missing[n & 1] = 1;
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    if (turn)
    #pragma unroll 1
                        for (int i = 0; i < C8; ++i) {
                            uint4 *x = reinterpret_cast<uint4 *>(place(u0 / C8 + i * (256 / C8)));
                            *x = make_uint4(x->x ^ turn, x->y ^ turn, x->z ^ turn, x->w ^ turn);
                        }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_q);
                    asm volatile("bar.sync 1, 256;" ::: "memory");  // (s_missing; the part before is through with its s_poison)
                    if (tid == 128) s_missing[(n + 1) & 1] = s_poison[(n + 1) & 1] = 0;
                }
            }
            const int nq = g.n_tok > per ? 2 : 1;
            const bool dual = nq == 1 && g.n_kt > 1;
            float m = -CUDART_INF_F, l = 0.f;
            const int row_q = dual ? 0 : q, p = row_q * per + r / gq;
            if (dual || q < nq) {
                const int pos = g.pos0 + min(p, g.n_tok - 1);
                // columns (positions from g.base on) that this row sees, that all rows of the unit see, that some row sees
                const int hi = g.causal ? pos + 1 - g.base : g.keys, all_hi = g.causal ? g.pos0 + 1 - g.base : g.keys;
                const bool missing = !dry && s_missing[n & 1] != 0;
                auto huge = [&] { if (fabsf(m) > kWpHuge<T> && m != -CUDART_INF_F && opaque(!dry)) s_poison[n & 1] = 1; };
#pragma unroll 1
                for (int j = dual ? q : 0; j < g.n_kt; j += dual ? 2 : 1) {
                    const int i = i0 + j, c0 = kPfKeys * (g.t0 + j);
                    const bool fresh = opaque(j < (dual ? 2 : 1)), run = opaque(!dry);
                    uint32_t valid = 0xffu;  // blocks that are there
                    bool part = c0 + kPfKeys > all_hi;
                    if (opaque(missing)) {
#pragma unroll 1
                        for (int b = 0; b < 8; ++b) {
                            const int u = 8 * (g.t0 + j) + b, col = ((g.base >> 4) + u) >> bpp;
                            const int page = col < a.c.max_pages ? a.c.table[(size_t)g.seq * a.c.max_pages + col] : -1;
                            if (page < 0 || page >= a.c.n_pages) valid &= ~(1u << b);
                        }
                        part = part || valid != 0xffu;
                    }
                    if (part && opaque(dual || q == 0)) {  // thread = V row: those that nobody sees become zero, the others are looked through
                        wp_wait(b_full + 8 * (i & 3), i >> 2, abortp, a.polls);
                        const int cc = c0 + r;
                        uint8_t *row = sv + (i & 1) * NB * KB + r * 128;
                        if (!kHalf && (valid >> (r >> 4) & 1u) && cc < all_hi) {
                            // (seen by every row: whatever it is, it belongs in every result)
                        } else if ((valid >> (r >> 4) & 1u) && cc < g.keys) {
                            // an exponent of ones (what is no number) and one more carries into the sign's place
                            constexpr uint32_t E = kHalf ? 0x7c007c00u : 0x7f807f80u, ONE = E & ~(E << 1);
                            uint32_t odd = 0u;
#pragma unroll 2
                            for (int d = 0; d < DH / 8; ++d) {
                                const uint4 y = *reinterpret_cast<const uint4 *>(row + (d >> 3) * KB + (((d & 7) ^ (r & 7)) * 16));
                                odd |= ((y.x & E) + ONE) | ((y.y & E) + ONE) | ((y.z & E) + ONE) | ((y.w & E) + ONE);
                            }
                            if (odd & 0x80008000u) s_poison[n & 1] = 1;
                        } else {
#pragma unroll 2
                            for (int d = 0; d < DH / 8; ++d) *reinterpret_cast<uint4 *>(row + (d >> 3) * KB + (((d & 7) ^ (r & 7)) * 16)) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    if (run) wp_wait(b_s + 8 * q, count++, abortp, a.polls);
                    __syncwarp();
                    tc_fence_after();
                    uint32_t s[4][32];
#pragma unroll
                    for (int x = 0; x < 4; ++x) wp_ld32(t_s + 32 * x, s[x]);
                    wp_ld_wait();
#pragma unroll
                    for (int x = 0; x < 4; ++x) wp_pin(s[x]);
                    if (part) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t there = (valid >> (2 * x) & 1u ? 0xffffu : 0u) | (valid >> (2 * x + 1) & 1u ? 0xffff0000u : 0u);
                            const uint32_t see = bits_between(0, hi - c0 - 32 * x) & there;
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[x][e] = see >> e & 1u ? s[x][e] : 0xff800000u;  // -inf
                        }
                    }
                    uint64_t sum;
                    uint32_t w[32];
                    // A probability that f16 has no number for would make 0 x inf of an infinite value: where every row sees every key it counts as 2^-24
                    // (2^-31 of the row's largest); tiles in parts are looked through.
                    const uint32_t least = part ? 0u : 0x00010001u;
                    const uint64_t c2 = f2_pack(c, c);
                    auto top = [&] {
                        float x[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                        for (int y = 0; y < 4; ++y)
#pragma unroll
                            for (int e = 0; e < 32; e += 2) x[(e >> 1) & 3] = max3_nan(x[(e >> 1) & 3], __uint_as_float(s[y][e]), __uint_as_float(s[y][e + 1]));
                        return max3_nan(max3_nan(x[0], x[1], x[2]), x[3], x[3]) * c;
                    };
                    const float mx = top();
                    bool grow;
                    float corr;
                    if constexpr (kHalf) {  // (by the difference, which is exact where the two are near: no rounding of a large m makes P infinite)
                        grow = fresh || (!(mx - fmaxf(m, -3e38f) <= kWpLazy + kWpBelow) && !(m != m));
                        corr = grow && !fresh ? ex2(m - (mx - kWpBelow)) : 1.f;
                    } else {
                        grow = fresh || (!(mx <= m + kWpLazy) && !(m != m));  // (a maximum that is no number stays)
                        corr = grow && !fresh ? ex2(m - mx) : 1.f;
                    }
                    if (__any_sync(0xffffffffu, grow)) {
                        if (grow) m = mx < CUDART_INF_F ? (kHalf ? mx - kWpBelow : mx) : CUDART_NAN_F;  // (inf - inf, as the formula has it)
                        huge();
                        l *= corr;
                        if (!fresh) {  // (the MMAs that wrote O are complete: S of these keys was issued behind them)
#pragma unroll 1
                            for (int d = 0; d < DH; d += 32) {
                                uint32_t o[32];
                                wp_ld32(t_o + d, o);
                                wp_ld_wait();
                                wp_pin(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
                                tc_st32(t_o + d, o);
                            }
                        }
                    }
                    const float base = m == -CUDART_INF_F ? 0.f : m;
                    sum = 0ull;
                    wp_exps<T>(s[0], s[1], c2, f2_pack(-base, -base), least, sum, w);
                    auto hand_over = [&](int h) {
                        tc_st32(t_s + 32 * h, w);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0 && run) mbar_arrive(b_p + 8 * (2 * q + h));
                    };
                    hand_over(0);
                    wp_pin(s[2]);  // (no probability of the second half before the first is handed over)
                    wp_pin(s[3]);
                    wp_exps<T>(s[2], s[3], c2, f2_pack(-base, -base), least, sum, w);
                    hand_over(1);
                    float l0, l1;
                    f2_unpack(sum, l0, l1);
                    l += l0 + l1;
                }
                if (dry) continue;
                wp_wait(b_o + 8 * q, ended++, abortp, a.polls);
                __syncwarp();
                tc_fence_after();
            }
            i0 += g.n_kt;
            // ---- the rows go out: parts as they stand in tensor memory, four dims of all rows after four dims of all rows; results through the place of Q,
            // whole lines at a time
            constexpr int CH = DH / 8;  // 16-byte chunks of a row in T
            float4 *const swap = reinterpret_cast<float4 *>(sq) + r;  // [DH / 4][128 rows]: the second stream's O
            auto load_o = [&](int d, uint32_t (&o)[32]) {
                wp_ld32(t_o + d, o);
                wp_ld_wait();
                wp_pin(o);
            };
            if (dual) {
                asm volatile("bar.sync 1, 256;" ::: "memory");  // (both streams' MMAs are complete: Q is no longer read)
                if (q == 1) {
                    s_ml[r] = make_float2(m, l);
#pragma unroll 1
                    for (int d = 0; d < DH; d += 32) {
                        uint32_t o[32];
                        load_o(d, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            swap[(d / 4 + e) * kWpRows] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
            if (q < nq) {
                float f0 = 1.f, f1 = 0.f;
                bool none1 = true;
                const bool none0 = m == -CUDART_INF_F;  // (no key seen: O may be 0 x whatever)
                if (dual) {
                    const float2 other = s_ml[r];
                    none1 = other.x == -CUDART_INF_F;
                    const float t = none0 ? other.x : none1 ? m : m > other.x ? m : other.x, base = t == -CUDART_INF_F ? 0.f : t;
                    f0 = none0 ? 0.f : ex2(m - base);
                    f1 = none1 ? 0.f : ex2(other.x - base);
                    l = l * f0 + other.y * f1;
                    if (m != m || other.x != other.x) f0 = f1 = l = CUDART_NAN_F;
                    m = t;
                }
                const bool direct = g.row < 0;
                if (direct) {
                    const float inv = none0 && none1 ? 0.f : 1.f / l;
                    f0 *= inv;
                    f1 *= inv;
                }
                const int rows = min(per, g.n_tok - row_q * per) * gq, R = g.n_tok * gq, first = row_q * per * gq;  // of this tile; of the part; before this tile
                const bool store = r < rows && !*abortp;
                if (!direct && store) a.ml[g.row + first + r] = make_float2(m, l);
                float4 *const part = reinterpret_cast<float4 *>(a.o + g.row * DH) + first + r;
                auto chunk = [&](int row, int x) { return reinterpret_cast<uint4 *>(sq + q * NB * QB) + row * CH + (x ^ (row & (CH - 1))); };
                uint4 *const mine = reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + ((size_t)(g.tok0 + min(p, g.n_tok - 1)) * a.p.Hq + g.kvh * gq + r % gq) * DH);
#pragma unroll 1
                for (int d = 0; d < DH; d += 32) {
                    uint32_t o[32];
                    load_o(d, o);
                    float y[32];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 x = dual && !none1 ? swap[(d / 4 + e) * kWpRows] : make_float4(0.f, 0.f, 0.f, 0.f);
                        const float z[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) y[4 * e + k] = (none0 ? 0.f : __uint_as_float(o[4 * e + k]) * f0) + z[k] * f1;
                    }
                    if (direct) {  // (of dual rows, straight away: the place of Q holds other rows' second half still)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!dual || store) *(dual ? mine + d / 8 + e : chunk(r, d / 8 + e)) = make_uint4(pack_pair<T>(y[8 * e], y[8 * e + 1]), pack_pair<T>(y[8 * e + 2], y[8 * e + 3]), pack_pair<T>(y[8 * e + 4], y[8 * e + 5]), pack_pair<T>(y[8 * e + 6], y[8 * e + 7]));
                    } else if (store) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) part[(int64_t)(d / 4 + e) * R] = make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
                    }
                }
                if (direct && !dual) {
                    __syncwarp();
                    const int lr = lane / CH, lc = lane % CH;
                    if (!*abortp)
#pragma unroll 4
                        for (int x = 0; x < 32; x += 32 / CH) {
                            const int rr = 32 * (warp & 3) + x + lr, pp = rr * inv_gq >> 16;
                            if (rr < rows)
                                *reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + ((size_t)(g.tok0 + row_q * per + pp) * a.p.Hq + g.kvh * gq + rr - pp * gq) * DH + 8 * lc) = *chunk(rr, lc);
                        }
                }
                tc_fence_before();
            }
        }
    }
    __syncwarp();
    if (*abortp) {  // a wait ran out: what this CTA has asked for lands within microseconds; do not leave before
#pragma unroll 1
        for (int i = 0; i < 64; ++i) __nanosleep(4000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tc_dealloc(tmem, 512u);
    }
    const bool gave_up = *abortp != 0;
    if (tid == 0 && (gave_up || s_no_page)) flag(a.status, gave_up ? RIVER_E_TIMEOUT : RIVER_E_BADARG);
}

// (the head dim of 64 asks for as much as 128 does: no CTA that wants tensor memory shares an SM with one that holds all of it)
inline size_t prefix_tiles_smem() { return 1024 + 7 * 2 * 128 * 128; }

}  // namespace river

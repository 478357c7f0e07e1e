// Attention over shared prefixes: a sequence's own positions for single tokens, and the joining of parts (sm_100a, internal).
//
// prefix_step_kernel: a cluster owns one query token and up to eight query heads of one KV head; its CTAs share out the blocks of 16 positions
// from the first one that is the sequence's own up to the token's, a warp takes every fourth block of its CTA.  Everything stays in registers, as in
// the windowed kernel of single tokens (window_attn_step.cuh): S = Q K^T and O^T += V^T P^T by mma.sync m16n8k16, whose operands are the rows as they
// were loaded, P = hi + lo.  What the kernel of the groups' keys has left of a row joins at the end, shared out over the cluster like the positions:
// the kernel starts beside that one and waits for it only there.
// Bound by HBM where rows are many.
#pragma once
#include "prefix_units.cuh"
#include "window_attn_step.cuh"

namespace river {

// Parts of one row's unit that the scratch holds: lane k gets the first row (of the token's heads) of the part of CTA c0 + k, -1 where that has none.
__device__ __forceinline__ int64_t pf_part_row(const PrefixArgs &a, const PfHead &h, int64_t x, const PfUnit &u, int kvh, int token, bool group, int c) {
    if (c >= a.p.ctas || (int64_t)c * h.share >= x + u.w) return -1;
    const PfPart p = pf_part(a.p, h.share, x, u, c, kvh, group);
    return p.k1 > p.k0 && p.row >= 0 ? p.row + (int64_t)(token - u.tok) * a.p.gq : -1;
}
// The unit of a group's keys that has this token; whether there is one
__device__ __forceinline__ bool pf_group_unit(const PrefixArgs &a, int seq, int token, int kvh, int span, const PfHead &h, PfUnit &u, int64_t &x) {
    const int l = a.lead[seq];
    if (l < 0 || l > seq || h.share < 1) return false;
    const PfGroup g = a.group[l];
    if (g.tok0 < 0 || g.tok0 > token || g.keys < 1 || g.at < 0 || g.at >= h.all) return false;  // (what stands there where lead is no first sequence)
    u = pf_unit(pf_group_entry(g.tok0, a.p.n_tokens - g.tok0, l, g.keys, span), (token - g.tok0) / span, span);  // (its rows behind the token do not matter here)
    x = kvh * h.all + g.at + u.at;
    return true;
}
// Adds to (m, l, acc) of a row - lane = DH / 32 dims - its parts in the scratch: of the CTAs c0 + k, k = first, first + step, ...  All lanes of a warp.
template <int DH>
__device__ __forceinline__ void pf_join(const PrefixArgs &a, const PfHead &h, int64_t x, const PfUnit &u, int kvh, int g, int token, bool group, int first, int step,
                                        float &m, float &l, float (&acc)[DH / 32]) {
    constexpr int E = DH / 32;
    const int lane = threadIdx.x & 31;
    const int c0 = (int)(x / h.share), c1 = (int)min((int64_t)a.p.ctas, (x + u.w - 1) / h.share + 1);
    for (int b = c0 + first; b < c1; b += 32 * step) {
        const int64_t row = pf_part_row(a, h, x, u, kvh, token, group, b + lane * step);
        const float2 ml = row >= 0 ? a.ml[row + g] : make_float2(-CUDART_INF_F, 0.f);
        float top = ml.x;
        bool odd = ml.x != ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        odd = __any_sync(0xffffffffu, odd);
        top = odd ? CUDART_NAN_F : fmaxf(top, m);
        if (top == -CUDART_INF_F) continue;
        const float old = m == -CUDART_INF_F ? 0.f : ex2(m - top), f = ml.x == -CUDART_INF_F ? 0.f : ex2(ml.x - top);
        m = top;
        l = l * old + warp_sum(ml.y * f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= old;
        unsigned have = __ballot_sync(0xffffffffu, f != 0.f);  // (a part without a visible key holds zeros)
        while (have) {
            float v[4][E], w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int src = have ? __ffs(have) - 1 : 0;
                const int64_t rr = __shfl_sync(0xffffffffu, row, src);
                const float ff = __shfl_sync(0xffffffffu, f, src);
                w[k] = have ? ff : 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) v[k][e] = 0.f;
                if (have) {
                    const float *p = a.o + (rr + g) * DH + E * lane;
                    if constexpr (E == 4) {
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(p));
                        v[k][0] = y.x; v[k][1] = y.y; v[k][2] = y.z; v[k][3] = y.w;
                    } else {
                        const float2 y = __ldcg(reinterpret_cast<const float2 *>(p));
                        v[k][0] = y.x; v[k][1] = y.y;
                    }
                }
                have &= have - 1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += v[k][e] * w[k];
        }
    }
}
template <class T, int DH>
__device__ __forceinline__ void pf_store(T *out, float l, const float (&acc)[DH / 32]) {  // out: of this lane
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < DH / 32; e += 2) *reinterpret_cast<uint32_t *>(out + e) = pack_pair<T>(acc[e] * inv, acc[e + 1] * inv);
}

// grid: splits x (Hkv * tiles of eight heads) x (max_q * n_seqs), linear, clusters of `splits`.  a.p.groups 0: the sequences' positions from the first on
template <class T, int DH>
__global__ void __launch_bounds__(32 * kStepWarps, kStepCtas) prefix_step_kernel(const PrefixArgs a, int splits) {
    namespace cg = cooperative_groups;
    constexpr int C = DH / 32, H = DH / 64;  // 16-byte chunks of a K row per lane; of a V row
    __shared__ float s_o[kStepWarps][8][DH];
    __shared__ float2 s_ml[kStepWarps][8];
    __shared__ float s_c[8][DH];
    __shared__ float2 s_cml[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int gq = a.p.gq, rt = (gq + 7) / 8, split = blockIdx.x % splits;
    const int unit = blockIdx.x / splits, tile = unit % (a.c.Hkv * rt), row = unit / (a.c.Hkv * rt);
    const int kvh = tile / rt, head0 = kvh * gq + tile % rt * 8, heads = min(8, gq - tile % rt * 8);
    const int seq = row / a.max_q, i = row % a.max_q;
    const int tok0 = a.q_start[seq], end = a.q_start[seq + 1], held = a.c.lens[seq], told = a.p.groups ? a.shared[seq] : 0;
    const bool odd = tok0 < 0 || end < tok0 || end > a.p.n_tokens;
    if (!a.p.groups && split == 0 && tile == 0 && i == 0 && threadIdx.x == 0 && !pf_sound(a, seq)) flag(a.status, RIVER_E_BADARG);  // (else the groups' kernel tells)
    if (odd || i >= end - tok0) {
        pdl_wait();
        return;
    }
    const int n = end - tok0, token = tok0 + i, pos = pf_len(a.c, held) - n + i, base = pf_shared(a.c, told);
    T *out = static_cast<T *>(a.out) + ((size_t)token * a.p.Hq + head0) * DH;
    // blocks of 16 positions: base / 16 .. pos / 16
    const int wb0 = base >> 4, nb = pos < base ? 0 : (pos >> 4) - wb0 + 1, b0 = (int)((int64_t)nb * split / splits), b1 = (int)((int64_t)nb * (split + 1) / splits);

    uint4 q[C];
    const T *qp = static_cast<const T *>(a.q) + token * a.q_tok + (head0 + g) * a.q_head + 8 * t;
#pragma unroll
    for (int c = 0; c < C; ++c) q[c] = g < heads ? *reinterpret_cast<const uint4 *>(qp + 32 * c) : make_uint4(0u, 0u, 0u, 0u);

    const int32_t *tbl = a.c.table + (size_t)seq * a.c.max_pages;
    const int bpp = a.c.ps_log2 - 4;  // log2 of a page's blocks
    auto page_of = [&](int u) {  // -1: nothing there
        if (u >= b1) return -1;
        const int col = (wb0 + u) >> bpp, page = col < a.c.max_pages ? tbl[col] : -1;
        if (page < 0 || page >= a.c.n_pages) { flag(a.status, RIVER_E_BADARG); return -1; }
        return page;
    };
    const T *pool = reinterpret_cast<const T *>(a.c.pool);
    const size_t v_off = ((size_t)a.c.Hkv << a.c.ps_log2) * DH;
    uint4 kr[2][C], vr[4][H];
    auto load_k = [&](int b, int page) {
        const T *p = pool + a.c.row(a.layer0, page, 0, kvh, (b << 4) & ((1 << a.c.ps_log2) - 1)) + g * DH + 8 * t;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int c = 0; c < C; ++c) kr[x][c] = ldg_stream16(p + x * 8 * DH + 32 * c);
    };
    auto load_v = [&](int b, int page) {
        const T *p = pool + a.c.row(a.layer0, page, 0, kvh, (b << 4) & ((1 << a.c.ps_log2) - 1)) + v_off + 8 * g;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int key = 2 * t + (x & 1) + 8 * (x >> 1);
            const bool on = page >= 0 && 16 * b + key <= pos;
#pragma unroll
            for (int h = 0; h < H; ++h) vr[x][h] = on ? ldg_stream16(p + key * DH + 64 * h) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    float o[DH / 16][4], m = -CUDART_INF_F, l = 0.f;  // m, l: of head g (l: this lane's share)
#pragma unroll
    for (int x = 0; x < DH / 16; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] = 0.f;

    int u = b0 + warp, k = 0, pages = page_of(u + kStepWarps * lane), page = __shfl_sync(0xffffffffu, pages, 0);
    if (u < b1) {
        if (page >= 0) load_k(wb0 + u, page);
        load_v(wb0 + u, page);
    }
    for (; u < b1; u += kStepWarps) {
        const int b = wb0 + u;
        float s[2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x][e] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                mma_16<T>(s[x], q[c].x, 0u, q[c].y, 0u, kr[x][c].x, kr[x][c].y);
                mma_16<T>(s[x], q[c].z, 0u, q[c].w, 0u, kr[x][c].z, kr[x][c].w);
            }
        }
        if (++k == 32) {
            pages = page_of(u + kStepWarps * (1 + lane));
            k = 0;
        }
        const int next = __shfl_sync(0xffffffffu, pages, k);
        const bool more = u + kStepWarps < b1;
        if (more && next >= 0) load_k(b + kStepWarps, next);
        // scores of head g, keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        float p[4];
        const bool whole = page >= 0 && 16 * b + 15 <= pos;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            p[x] = s[x >> 1][x & 1] * a.scale_log2;
            if (!whole && (page < 0 || 16 * b + 2 * t + (x & 1) + 8 * (x >> 1) > pos)) p[x] = -CUDART_INF_F;
        }
        float mx = fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        mx = fmaxf(mx, m);
        if (__any_sync(0xffffffffu, mx > m)) {
            const float corr = mx > m ? ex2(m - mx) : 1.f;
            m = mx;
            l *= corr;
            const float c0 = __shfl_sync(0xffffffffu, corr, 8 * t), c1 = __shfl_sync(0xffffffffu, corr, 8 * t + 4);
#pragma unroll
            for (int x = 0; x < DH / 16; ++x) { o[x][0] *= c0; o[x][1] *= c1; o[x][2] *= c0; o[x][3] *= c1; }
        }
        const float top = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int x = 0; x < 4; ++x) p[x] = ex2(p[x] - top) * kStepScale<T>;
        l += (p[0] + p[1]) + (p[2] + p[3]);
        uint32_t hi0, lo0, hi1, lo1;
        split_pair<T>(p[0], p[1], hi0, lo0);
        split_pair<T>(p[2], p[3], hi1, lo1);
        // dims of an MMA's rows g, g + 8: dh 128: 8 g + x, 64 + 8 g + x (x < 8); dh 64: 8 g + x, 8 g + 4 + x (x < 4)
#pragma unroll
        for (int x = 0; x < DH / 16; ++x) {
            uint32_t w[4][2];  // [key][row g, row g + 8]: the word that holds the dim
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t v0[4] = {vr[e][0].x, vr[e][0].y, vr[e][0].z, vr[e][0].w};
                const uint32_t v1[4] = {vr[e][H - 1].x, vr[e][H - 1].y, vr[e][H - 1].z, vr[e][H - 1].w};
                w[e][0] = v0[x >> 1];
                w[e][1] = DH == 128 ? v1[x >> 1] : v1[2 + (x >> 1)];
            }
            const uint32_t sel = x & 1 ? 0x7632u : 0x5410u;
            const uint32_t a0 = __byte_perm(w[0][0], w[1][0], sel), a1 = __byte_perm(w[0][1], w[1][1], sel),
                           a2 = __byte_perm(w[2][0], w[3][0], sel), a3 = __byte_perm(w[2][1], w[3][1], sel);
            mma_16<T>(o[x], a0, a1, a2, a3, hi0, hi1);
            mma_16<T>(o[x], a0, a1, a2, a3, lo0, lo1);
        }
        page = next;
        if (more) load_v(b + kStepWarps, page);
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    // (O and l are held times kStepScale: that goes into the maximum, as the other parts have none)
    if (t == 0) s_ml[warp][g] = make_float2(std::is_same<T, __half>::value ? m - 15.f : m, l);
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
        constexpr int R = DH == 128 ? 8 : 4;  // consecutive dims of a row set
        float *d = &s_o[warp][2 * t + hh][8 * g];
#pragma unroll
        for (int x = 0; x < R; x += 4) {
            *reinterpret_cast<float4 *>(d + x) = make_float4(o[x][hh], o[x + 1][hh], o[x + 2][hh], o[x + 3][hh]);
            *reinterpret_cast<float4 *>(d + (DH == 128 ? 64 : 4) + x) = make_float4(o[x][2 + hh], o[x + 1][2 + hh], o[x + 2][2 + hh], o[x + 3][2 + hh]);
        }
    }
    pdl_wait();  // (the groups' parts)
    PfUnit gu = {};
    PfHead head = {};
    int64_t gx = 0;
    bool joins = base > 0;
    if (joins) {
        head = *a.head;
        joins = pf_group_unit(a, seq, token, kvh, 2 * pf_per(gq), head, gu, gx);
    }
    __syncthreads();
    // the warps' parts, and this CTA's share of the groups': a warp per head, lane = dims
    constexpr int E = DH / 32;
    for (int h = warp; h < heads; h += kStepWarps) {
        float mm = -CUDART_INF_F, ll = 0.f, acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) mm = fmaxf(mm, s_ml[w][h].x);
        const float mb = mm == -CUDART_INF_F ? 0.f : mm;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) {
            const float2 x = s_ml[w][h];
            const float f = ex2(x.x - mb);
            ll += x.y * f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += s_o[w][h][E * lane + e] * f;
        }
        if (joins) pf_join<DH>(a, head, gx, gu, kvh, head0 - kvh * gq + h, token, true, split, splits, mm, ll, acc);
        if (splits == 1) {
            pf_store<T, DH>(out + h * DH + E * lane, ll, acc);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) s_c[h][E * lane + e] = acc[e];
            if (lane == 0) s_cml[h] = make_float2(mm, ll);
        }
    }
    if (splits == 1) return;
    // the cluster's parts: every CTA finishes its share of the heads' dims
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int x = split * 32 * kStepWarps + threadIdx.x; x < heads * DH / 2; x += splits * 32 * kStepWarps) {  // pairs of dims
        const int e = 2 * x, hd = e / DH, d = e % DH;
        float2 ml[kStepMaxSplits], v[kStepMaxSplits];
        float top = -CUDART_INF_F;
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) {
            ml[r] = make_float2(-CUDART_INF_F, 0.f);
            v[r] = make_float2(0.f, 0.f);
            if (r < splits) {
                ml[r] = *cluster.map_shared_rank(&s_cml[hd], r);
                v[r] = *reinterpret_cast<const float2 *>(cluster.map_shared_rank(&s_c[hd][d], r));
            }
        }
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) top = fmaxf(top, ml[r].x);
        const float tb = top == -CUDART_INF_F ? 0.f : top;
        float sum = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) {
            const float f = ex2(ml[r].x - tb);
            sum += ml[r].y * f;
            y0 += v[r].x * f;
            y1 += v[r].y * f;
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint32_t *>(out + e) = pack_pair<T>(y0 * inv, y1 * inv);
    }
    cluster.sync();  // (peers read this CTA's part)
}

// The sequence that has row `token`; -1: none
__device__ __forceinline__ int pf_seq_of(const PrefixArgs &a, int token) {
    int lo = 0, hi = a.c.n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_start[mid] <= token) lo = mid; else hi = mid;
    }
    return a.q_start[lo] <= token && token < a.q_start[lo + 1] && a.q_start[lo] >= 0 && a.q_start[lo + 1] <= a.p.n_tokens ? lo : -1;
}
// Rows with parts of both kinds, a warp per row: grid-stride over tokens x heads.
template <class T, int DH>
__global__ void __launch_bounds__(256) prefix_join_kernel(const PrefixArgs a) {
    const int gq = a.p.gq, span = 2 * pf_per(gq), lane = threadIdx.x & 31;
    pdl_wait();
    const PfHead h = *a.head;
    for (int64_t w = blockIdx.x * 8 + (threadIdx.x >> 5); w < (int64_t)a.p.n_tokens * a.p.Hq; w += gridDim.x * 8) {
        const int token = (int)(w / a.p.Hq), head = (int)(w % a.p.Hq), kvh = head / gq, seq = pf_seq_of(a, token);
        if (seq < 0) continue;
        float m = -CUDART_INF_F, l = 0.f, acc[DH / 32];
#pragma unroll
        for (int e = 0; e < DH / 32; ++e) acc[e] = 0.f;
        PfUnit u;
        int64_t x;
        if (pf_shared(a.c, a.shared[seq]) > 0 && pf_group_unit(a, seq, token, kvh, span, h, u, x)) pf_join<DH>(a, h, x, u, kvh, head - kvh * gq, token, true, 0, 1, m, l, acc);
        const PfEntry e = pf_entry(a, a.c.n_seqs + seq, span);
        u = pf_unit(e, (token - e.tok0) / span, span);
        pf_join<DH>(a, h, kvh * h.all + a.own_at[seq] + u.at, u, kvh, head - kvh * gq, token, false, 0, 1, m, l, acc);
        pf_store<T, DH>(static_cast<T *>(a.out) + w * DH + DH / 32 * lane, l, acc);
    }
}
// Sequences' units that were cut: block (c, y) has the unit that the end of CTA c's part cuts, if it is the first cut in there, and every kJoinBlocks-th
// eight rows of it.
constexpr int kJoinBlocks = 8;
template <class T, int DH>
__global__ void __launch_bounds__(256) prefix_join_cut_kernel(const PrefixArgs a) {
    const int gq = a.p.gq, span = 2 * pf_per(gq), lane = threadIdx.x & 31;
    pdl_wait();
    const PfHead h = *a.head;
    const int64_t cut = (blockIdx.x + 1) * h.share;
    if (cut >= h.all * a.c.Hkv) return;
    const int kvh = (int)(cut / h.all);
    const int64_t y = cut - kvh * h.all;
    int lo = 0, hi = a.c.n_seqs;  // the last sequence that begins at or before y (those without units weigh nothing)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.own_at[mid] <= y) lo = mid; else hi = mid;
    }
    const PfEntry e = pf_entry(a, lo, span);
    if (e.w == 0) return;
    const int64_t at = a.own_at[lo];
    const PfUnit u = pf_unit(e, pf_unit_at(e, y - at, span), span);
    const int64_t x = kvh * h.all + at + u.at;
    if (x == cut || (int64_t)blockIdx.x * h.share > x) return;  // (not cut here, or cut before)
    if (pf_part(a.p, h.share, x, u, (int)((x + u.w - 1) / h.share), kvh, false).row < 0) return;  // (its last CTA has every tile)
    for (int r = blockIdx.y * 8 + (threadIdx.x >> 5); r < u.n * gq; r += 8 * kJoinBlocks) {
        const int token = u.tok + r / gq, g = r % gq;
        float m = -CUDART_INF_F, l = 0.f, acc[DH / 32];
#pragma unroll
        for (int z = 0; z < DH / 32; ++z) acc[z] = 0.f;
        pf_join<DH>(a, h, x, u, kvh, g, token, false, 0, 1, m, l, acc);
        pf_store<T, DH>(static_cast<T *>(a.out) + ((size_t)token * a.p.Hq + kvh * gq + g) * DH + DH / 32 * lane, l, acc);
    }
}

}  // namespace river

// Windowed attention of single tokens: split over the visible positions and joined inside a cluster (sm_100a, internal).
//
// A cluster owns one query token and up to eight query heads of one KV head; its CTAs share out the visible blocks of 16 positions
// (those of the sinks, then those of the window), a warp takes every fourth block of its CTA.  Everything stays in registers:
//   S [8 heads x 16 keys] = Q K^T      mma.sync m16n8k16, rows = heads (the upper eight are zero).  Products of a sum may come in any order,
//                                      so a lane's 16 consecutive bytes of a key row are the B operand of two steps as they are loaded, and
//                                      Q is loaded in the same order: no shared memory, no transposition.
//   softmax                            online, fp32, base 2: a row lies with four lanes.
//   O^T [dh x 8 heads] += V^T P^T      S in its accumulator layout is the B operand; the A operand pairs the values of two keys, which a
//                                      byte permutation makes of two loaded rows.  P = hi + lo, so that it keeps 16 bits and more (f16:
//                                      kStepScale; down to 2^-23 of the row's largest; what is not 0 counts as 2^-38 at least).
// K of the next block is requested when S has been computed, V when O has: 8 KB (dh 128) per warp are under way all the time.
//
// Bound by HBM where rows are many: 128 rows of the 8B class, window 8192, 4.2 GB in 650 to 685 us by the GPU (6.1 to 6.45 TB/s, the copy rate); one row by
// its chain (1B class, window 1024: 5.4 us without the host): lengths, page ids, K, then the warps' and the CTAs' parts joined.
//
// Hidden positions: their scores are -inf and their values are zero in the operand (never loaded), so what the pool holds there
// does not matter.  hi is rounded downwards from a little below p, and both are at least the type's smallest number where p is not 0: an
// infinite value that is seen gives infinity and not 0 x inf.
#pragma once
#include <cooperative_groups.h>

#include <type_traits>

#include "window_attn_rows.cuh"

namespace river {

constexpr int kStepWarps = 4;
constexpr int kStepCtas = 3;         // resident per SM (168 registers)
constexpr int kStepMaxSplits = 16;   // CTAs of a cluster
// P and its sum are held times kStepScale: f16 ends at 2^-24 below and 2^16 above, and p at most 1 would leave the upper part unused (32768 positions
// of 2^-25 each counted in the sum but not in O).  bf16 has fp32's exponents.
template <class T> constexpr float kStepScale = std::is_same<T, __half>::value ? 32768.f : 1.f;

template <class T> __device__ __forceinline__ void mma_16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma_16<__nv_bfloat16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma_16<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// p -> hi (rounded towards zero from p (1 - 2^-9)) and lo = p - hi > 0, two values to a word; f16: both at least 2^-24 where p is not 0
template <class T> __device__ __forceinline__ void split_pair(float p0, float p1, uint32_t &hi, uint32_t &lo);
template <> __device__ __forceinline__ void split_pair<__nv_bfloat16>(float p0, float p1, uint32_t &hi, uint32_t &lo) {
    const uint32_t h0 = __float_as_uint(p0 * 0.998046875f) & 0xffff0000u, h1 = __float_as_uint(p1 * 0.998046875f) & 0xffff0000u;
    hi = (h0 >> 16) | h1;
    const __nv_bfloat162 l = __floats2bfloat162_rn(p0 - __uint_as_float(h0), p1 - __uint_as_float(h1));
    lo = *reinterpret_cast<const uint32_t *>(&l);
}
template <> __device__ __forceinline__ void split_pair<__half>(float p0, float p1, uint32_t &hi, uint32_t &lo) {
    const float least0 = p0 > 0.f ? 1.f / 16777216.f : 0.f, least1 = p1 > 0.f ? 1.f / 16777216.f : 0.f;  // 2^-24
    const __half2 h = __halves2half2(__float2half_rz(fmaxf(p0 * 0.998046875f, least0)), __float2half_rz(fmaxf(p1 * 0.998046875f, least1)));
    const __half2 l = __floats2half2_rn(fmaxf(p0 - __low2float(h), least0), fmaxf(p1 - __high2float(h), least1));
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = *reinterpret_cast<const uint32_t *>(&l);
}
template <class T> __device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float a, float b) {
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}

// grid: splits x (Hkv * tiles of eight heads) x (max_q * n_seqs), linear, clusters of `splits`
template <class T, int DH>
__global__ void __launch_bounds__(32 * kStepWarps, kStepCtas) window_attn_step_kernel(const WindowArgs a, int splits) {
    namespace cg = cooperative_groups;
    constexpr int C = DH / 32, H = DH / 64;  // 16-byte chunks of a K row per lane; of a V row
    __shared__ float s_o[kStepWarps][8][DH];
    __shared__ float2 s_ml[kStepWarps][8];
    __shared__ float s_c[8][DH];
    __shared__ float2 s_cml[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int gq = a.Hq / a.c.Hkv, rt = (gq + 7) / 8, split = blockIdx.x % splits;
    const int unit = blockIdx.x / splits, tile = unit % (a.c.Hkv * rt), row = unit / (a.c.Hkv * rt);
    const int kvh = tile / rt, head0 = kvh * gq + tile % rt * 8, heads = min(8, gq - tile % rt * 8);
    const int seq = row / a.max_q, i = row % a.max_q;
    const int tok0 = a.q_start[seq], end = a.q_start[seq + 1], held = a.c.lens[seq];
    const bool odd = tok0 < 0 || end < tok0 || end > a.n_tokens;
    if (threadIdx.x == 0 && (odd || end - tok0 > a.max_q)) flag(a.status, RIVER_E_BADARG);
    if (odd || i >= end - tok0) return;
    const int n = end - tok0, len = window_len(a, held);
    const int token = tok0 + i, pos = len - n + i;
    T *out = static_cast<T *>(a.out) + ((size_t)token * a.Hq + head0) * DH;
    // blocks of 16 positions: n_sb of the sinks, then wb0 .. pos / 16
    const int low = window_low(pos, a.window), wb0 = low >> 4, n_sb = min((min(a.sinks, low) + 15) >> 4, wb0);
    const int nb = pos < 0 ? 0 : n_sb + (pos >> 4) - wb0 + 1, b0 = nb * split / splits, b1 = nb * (split + 1) / splits;

    uint4 q[C];
    const T *qp = static_cast<const T *>(a.q) + token * a.q_tok + (head0 + g) * a.q_head + 8 * t;
#pragma unroll
    for (int c = 0; c < C; ++c) q[c] = g < heads ? *reinterpret_cast<const uint4 *>(qp + 32 * c) : make_uint4(0u, 0u, 0u, 0u);

    const int32_t *tbl = a.c.table + (size_t)seq * a.c.max_pages;
    const int bpp = a.c.ps_log2 - 4;  // log2 of a page's blocks
    auto block_of = [&](int u) { return u < n_sb ? u : wb0 + u - n_sb; };
    auto page_of = [&](int u) {  // -1: nothing there
        if (u >= b1) return -1;
        const int col = block_of(u) >> bpp, page = col < a.c.max_pages ? tbl[col] : -1;
        if (page < 0 || page >= a.c.n_pages) { flag(a.status, RIVER_E_BADARG); return -1; }
        return page;
    };
    auto seen = [&](int j) { return j <= pos && (j < a.sinks || j >= low); };
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
            const bool on = page >= 0 && seen(16 * b + key);
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
        if (page >= 0) load_k(block_of(u), page);
        load_v(block_of(u), page);
    }
    for (; u < b1; u += kStepWarps) {
        const int b = block_of(u);
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
        if (more && next >= 0) load_k(block_of(u + kStepWarps), next);
        // scores of head g, keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        float p[4];
        const bool whole = page >= 0 && 16 * b + 15 <= pos && (16 * b >= low || 16 * b + 15 < a.sinks);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            p[x] = s[x >> 1][x & 1] * a.scale_log2;
            if (!whole && (page < 0 || !seen(16 * b + 2 * t + (x & 1) + 8 * (x >> 1)))) p[x] = -CUDART_INF_F;
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
        const float base = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int x = 0; x < 4; ++x) p[x] = ex2(p[x] - base) * kStepScale<T>;
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
        if (more) load_v(block_of(u + kStepWarps), page);
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (t == 0) s_ml[warp][g] = make_float2(m, l);
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
    __syncthreads();
    // the warps' parts: a warp per head, lane = dims
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
        if (splits == 1) {
            const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
            for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t *>(out + h * DH + E * lane + e) = pack_pair<T>(acc[e] * inv, acc[e + 1] * inv);
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
        const int e = 2 * x, head = e / DH, d = e % DH;
        float2 ml[kStepMaxSplits], v[kStepMaxSplits];
        float top = -CUDART_INF_F;
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) {
            ml[r] = make_float2(-CUDART_INF_F, 0.f);
            v[r] = make_float2(0.f, 0.f);
            if (r < splits) {
                ml[r] = *cluster.map_shared_rank(&s_cml[head], r);
                v[r] = *reinterpret_cast<const float2 *>(cluster.map_shared_rank(&s_c[head][d], r));
            }
        }
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) top = fmaxf(top, ml[r].x);
        const float tb = top == -CUDART_INF_F ? 0.f : top;
        float sum = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll
        for (int r = 0; r < kStepMaxSplits; ++r) {
            const float f = ex2(ml[r].x - tb);
            sum += ml[r].y * f;
            x0 += v[r].x * f;
            x1 += v[r].y * f;
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint32_t *>(out + e) = pack_pair<T>(x0 * inv, x1 * inv);
    }
    cluster.sync();  // (peers read this CTA's part)
}

// CTAs per cluster, by an estimate of the time in us.  A round of CTAs takes what HBM needs for its blocks, or 1.4 for each block
// that a warp has one after the other (a fetch and the products behind it), and 2 + s / 4 for its start and the joining.  Clusters of more
// than four leave places free: a GPC, of about 16 SMs, takes whole ones.  (8B-class heads, us with 3, 4, 6, 8, 16 CTAs: window 4096, 64
// rows 185, 184, 203, 218, 304; 16 rows 48, 67, 53, 61, 84; 4 rows 35, 28, 22, 19, 26; window 8192, one row 60, 47, 33, 27, 17.)
inline int step_splits(const WindowArgs &a, int num_sms, double &best_t) {
    const double tiles = (double)a.c.Hkv * ((a.Hq / a.c.Hkv + 7) / 8), units = (double)a.n_tokens * tiles;
    const double idle = std::max(0.0, (double)a.c.n_seqs * a.max_q - a.n_tokens) * tiles * 0.0015;  // places of queries that are none: a CTA each that leaves
    const int64_t cap = (int64_t)a.c.max_pages << a.c.ps_log2, blocks = (std::min<int64_t>(cap, (int64_t)a.window + a.sinks) >> 4) + 1;
    const double block_us = 64.0 * a.c.dh / 6.4e6;  // K and V of a block at 6.4 TB/s
    int best = 1;
    best_t = 1e300;
    for (int s = 1; s <= kStepMaxSplits; ++s) {
        const double places = s <= 4 ? num_sms * kStepCtas : num_sms / 18 * (16 * kStepCtas / s) * s;
        const double turns = 1.4 * (double)((blocks + s * kStepWarps - 1) / (s * kStepWarps)), stream = places * (double)blocks / s * block_us, fixed = 2.0 + 0.25 * s;
        const double rounds = units * s / places, full = std::floor(rounds), rest = rounds - full;
        const double t = full * (std::max(stream, turns) + fixed) + (rest > 0 ? std::max(stream * rest, turns) + fixed : 0.0) + idle * s;
        if (t < 0.99 * best_t) { best_t = t; best = s; }
    }
    return best;
}

}  // namespace river

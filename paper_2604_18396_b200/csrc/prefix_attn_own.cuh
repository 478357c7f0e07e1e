// Attention over shared prefixes: sequences' own positions for single tokens, and the joining of parts (sm_100a, internal).
#pragma once
#include "mma_sync.cuh"
#include "prefix_units.cuh"
#include "window_attn_prompt.cuh"

namespace river {

// A sequence's positions for single tokens: a cluster owns one query token and up to eight query heads of one KV head; its CTAs share out the blocks of 16
// positions from the sequence's own first one (without groups: from the first of all) to the token's, a warp takes every fourth block of its CTA.
//   K, V [16 x DH]             by TMA, boxes of 16 x 64, kPfDeep blocks of a warp under way: lists are short, and a block takes 1.5 to 4 us to come
//   S^T [16 keys x 8 heads]    = K Q^T: mma.sync m16n8k16, K by ldmatrix, Q in registers
//   softmax                    online, fp32, base 2: a lane has two heads of keys g, g + 8; the maximum is looked for in other lanes only where it has moved
//                              (bf16: by more than 2^8)
//   O^T [DH x 8 heads]         += V^T P^T: V by ldmatrix with transposition, P = hi + lo (16 bits and more; f16: kStepScale) by movmatrix
// Without groups the result is written, else O, not divided yet, its maximum and its sum go to the scratch; then this kernel starts beside the groups' one, on
// the SMs that one leaves free, and only its first CTA waits for it.
// Bound by HBM where lists are long: 128 rows of 8017 positions, 8 KV heads of 128, 4.21 GB in 612 us, 6.9 TB/s.  Of 256 rows with 50 to 1000 positions, 571 MB
// in 102 us, 5.6 TB/s; warps that stream equal shares of all rows' blocks took 138 (register loads) and 134 (cp.async).
// grid: splits x (Hkv * tiles of eight heads) x (max_q * n_seqs), linear, clusters of `splits`
constexpr int kPfDeep = 2;
template <int DH> constexpr int kPfOwnCtas = DH == 128 ? 3 : 4;  // resident per SM
template <int DH> constexpr size_t kPfOwnSmem = 1024 + (size_t)kStepWarps * kPfDeep * 64 * DH;

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <class T, int DH>
__global__ void __launch_bounds__(32 * kStepWarps, kPfOwnCtas<DH>) prefix_own_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ PrefixArgs a, int splits) {
    namespace cg = cooperative_groups;
    constexpr int NB = DH / 64, D = kPfDeep;  // boxes of a block's K or V
    constexpr bool kHalf = std::is_same<T, __half>::value;
    extern __shared__ uint8_t pf_raw[];
    __shared__ uint64_t bars[kStepWarps][D];
    __shared__ float2 s_ml[kStepWarps][8];
    __shared__ float s_c[8][DH];
    __shared__ float2 s_cml[8];
    __shared__ int s_abort;
    uint8_t *const rings = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(pf_raw) + 1023) & ~(uintptr_t)1023);
    float(*const s_o)[8][DH + 4] = reinterpret_cast<float(*)[8][DH + 4]>(rings);  // (when the blocks are through)
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int gq = a.p.gq, rt = (gq + 7) / 8, split = blockIdx.x % splits;
    const int unit = blockIdx.x / splits, tile = unit % (a.c.Hkv * rt), row = unit / (a.c.Hkv * rt);
    const int kvh = tile / rt, head0 = kvh * gq + tile % rt * 8, heads = min(8, gq - tile % rt * 8);
    const int seq = row / a.max_q, i = row % a.max_q;
    const bool direct = !a.p.groups;
    const int tok0 = a.q_start[seq], end = a.q_start[seq + 1], held = a.c.lens[seq], told = direct ? 0 : a.shared[seq];
    const bool odd = tok0 < 0 || end < tok0 || end > a.p.n_tokens;
    if (!direct) pdl_launch();
    auto leave = [&] { if (!direct && blockIdx.x == 0) pdl_wait(); };  // (this kernel ends behind the groups': who waits for it has both)
    if (direct && split == 0 && tile == 0 && i == 0 && threadIdx.x == 0 && !pf_sound(a, seq)) flag(a.status, RIVER_E_BADARG);  // (else the groups' kernel tells)
    if (odd || i >= end - tok0) return leave();
    const int n = end - tok0, token = tok0 + i, pos = pf_len(a.c, held) - n + i, base = pf_shared(a.c, told);
    const size_t out = (size_t)token * a.p.Hq + head0;  // first row
    // blocks of 16 positions: base / 16 .. pos / 16; this warp's: wb + 4 x, x < mine
    const int wb0 = base >> 4, nb = pos < base ? 0 : (pos >> 4) - wb0 + 1, b0 = (int)((int64_t)nb * split / splits), b1 = (int)((int64_t)nb * (split + 1) / splits);
    const int wb = wb0 + b0 + warp, mine = b1 - b0 > warp ? (b1 - b0 - warp + kStepWarps - 1) / kStepWarps : 0;

    const int32_t *tbl = a.c.table + (size_t)seq * a.c.max_pages;
    auto pages_from = [&](int x) {  // this lane's of the blocks x, x + 1, ..; -1: nothing there
        if (x + lane >= mine) return -1;
        const int col = (wb + kStepWarps * (x + lane)) >> (a.c.ps_log2 - 4), page = col < a.c.max_pages ? tbl[col] : -1;
        if (page < 0 || page >= a.c.n_pages) { flag(a.status, RIVER_E_BADARG); return -1; }
        return page;
    };
    int pages = pages_from(0), pages_next = -1;
    volatile int *abortp = &s_abort;
    const uint32_t bar = smem_u32(&bars[warp][0]), ring = smem_u32(rings) + warp * D * 64 * DH;
    if (lane == 0) {
        s_abort = 0;
#pragma unroll
        for (int x = 0; x < D; ++x) mbar_init(bar + 8 * x, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    auto ask = [&](int slot, int x, int page) {  // block x, on its way to a place of the ring
        if (lane == 0 && page >= 0) {
            const int r = ((page * 2 * a.c.Hkv + kvh) << a.c.ps_log2) + (((wb + kStepWarps * x) << 4) & ((1 << a.c.ps_log2) - 1));
            mbar_expect_tx(bar + 8 * slot, 64 * DH);
#pragma unroll
            for (int h = 0; h < NB; ++h) tma_load_2d(ring + slot * 64 * DH + 2048 * h, &tmap, 64 * h, r, bar + 8 * slot);
#pragma unroll
            for (int h = 0; h < NB; ++h) tma_load_2d(ring + slot * 64 * DH + 2048 * (NB + h), &tmap, 64 * h, r + (a.c.Hkv << a.c.ps_log2), bar + 8 * slot);
        }
    };
    // (a block whose page is missing uses no phase of its place's barrier: it is passed over)
#pragma unroll
    for (int x = 0; x < D; ++x) {
        const int page = __shfl_sync(0xffffffffu, pages, x);
        if (x < mine) ask(x, x, page);
    }
    uint32_t qb[DH / 16][2];  // dims 16 k + 2 t, + 1 and + 8, + 9 of head g
    const T *qp = static_cast<const T *>(a.q) + token * a.q_tok + (head0 + g) * a.q_head + 2 * t;
#pragma unroll
    for (int k = 0; k < DH / 16; ++k)
#pragma unroll
        for (int y = 0; y < 2; ++y) qb[k][y] = g < heads ? *reinterpret_cast<const uint32_t *>(qp + 16 * k + 8 * y) : 0u;
    float o[DH / 16][4];  // dims 16 d + g (+ 8) of heads 2 t, 2 t + 1
    float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, l0 = 0.f, l1 = 0.f;  // of heads 2 t, 2 t + 1 (the sums: of this lane's keys)
#pragma unroll
    for (int d = 0; d < DH / 16; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][e] = 0.f;
    constexpr float kSlack = kHalf ? 0.f : 8.f;  // (f16: P has no room above kStepScale)
    // where a lane's rows of ldmatrix begin: K rows lane & 15, V rows (lane & 7) + 8 (lane >> 4)
    const uint32_t k_row = (lane & 15) * 128, k_x = lane & 7, k_c = lane >> 4, v_row = ((lane & 7) + 8 * (lane >> 4)) * 128, v_c = lane >> 3 & 1;
    int slot = 0;
    uint32_t phases = 0;
#pragma unroll 1
    for (int x = 0; x < mine; ++x) {
        const int b = wb + kStepWarps * x;
        if ((x & 31) == 0) {
            if (x) pages = pages_next;
            pages_next = pages_from(x + 32);
        }
        const int page = __shfl_sync(0xffffffffu, pages, x & 31), ahead = __shfl_sync(0xffffffffu, (x & 31) + D < 32 ? pages : pages_next, (x + D) & 31);
        if (page >= 0) {
            wp_wait(bar + 8 * slot, phases >> slot, abortp, a.polls);
            __syncwarp();
            phases ^= 1u << slot;
            const uint32_t in = ring + slot * 64 * DH;
            float s[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[0][e] = s[1][e] = 0.f;
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                uint32_t f[4];
                ldsm_x4(f, in + (k >> 2) * 2048 + k_row + (((2 * (k & 3) + k_c) ^ k_x) << 4));
                mma_16<T>(s[k & 1], f[0], f[1], f[2], f[3], qb[k][0], qb[k][1]);
            }
            float p[4];  // key g: heads 2 t, 2 t + 1; key g + 8
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = (s[0][e] + s[1][e]) * a.scale_log2;
            const int hidden = 16 * b + 15 - pos;  // keys of this block behind the token
            if (hidden > 0) {
                if (g > 15 - hidden) p[0] = p[1] = -CUDART_INF_F;
                if (g + 8 > 15 - hidden) p[2] = p[3] = -CUDART_INF_F;
                // their values, whatever they are, become zero (nothing else is loaded into this place: it is the last block)
#pragma unroll 1
                for (int z = lane; z < hidden * NB * 8; z += 32) {
                    const uint32_t to = in + 2048 * NB + (z & 7) * 16 + (16 - hidden + (z >> 3) % hidden) * 128 + (z >> 3) / hidden * 2048;
                    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
                }
                __syncwarp();
            }
            const float x0 = fmaxf(p[0], p[2]), x1 = fmaxf(p[1], p[3]);
            if (__any_sync(0xffffffffu, x0 > m0 + kSlack || x1 > m1 + kSlack)) {
                float n0 = fmaxf(x0, m0), n1 = fmaxf(x1, m1);
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, y));
                    n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, y));
                }
                const float c0 = n0 > m0 ? ex2(m0 - n0) : 1.f, c1 = n1 > m1 ? ex2(m1 - n1) : 1.f;
                m0 = n0, m1 = n1;
                l0 *= c0, l1 *= c1;
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) { o[d][0] *= c0; o[d][1] *= c1; o[d][2] *= c0; o[d][3] *= c1; }
            }
            const float t0 = m0 == -CUDART_INF_F ? 0.f : m0, t1 = m1 == -CUDART_INF_F ? 0.f : m1;
            p[0] = ex2(p[0] - t0) * kStepScale<T>;
            p[1] = ex2(p[1] - t1) * kStepScale<T>;
            p[2] = ex2(p[2] - t0) * kStepScale<T>;
            p[3] = ex2(p[3] - t1) * kStepScale<T>;
            l0 += p[0] + p[2];
            l1 += p[1] + p[3];
            uint32_t hi0, lo0, hi1, lo1;
            split_pair<T>(p[0], p[1], hi0, lo0);
            split_pair<T>(p[2], p[3], hi1, lo1);
            hi0 = movmatrix(hi0), hi1 = movmatrix(hi1), lo0 = movmatrix(lo0), lo1 = movmatrix(lo1);
#pragma unroll
            for (int d = 0; d < DH / 16; ++d) {
                uint32_t f[4];
                ldsm_x4_trans(f, in + 2048 * NB + (d >> 2) * 2048 + v_row + (((2 * (d & 3) + v_c) ^ k_x) << 4));
                mma_16<T>(o[d], f[0], f[1], f[2], f[3], hi0, hi1);
                mma_16<T>(o[d], f[0], f[1], f[2], f[3], lo0, lo1);
            }
            __syncwarp();  // (all lanes have read this place)
        }
        if (x + D < mine && !*abortp) ask(slot, x + D, ahead);
        slot = slot == D - 1 ? 0 : slot + 1;
    }
#pragma unroll
    for (int y = 4; y < 32; y <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, y);
        l1 += __shfl_xor_sync(0xffffffffu, l1, y);
    }
    // (O and l are held times kStepScale, other parts are not.  It is taken out of them, which is exact, and not out of the maximum: from 2^24 on that has no units.)
    constexpr float kUnscale = 1.f / kStepScale<T>;
    if (g == 0) {
        s_ml[warp][2 * t] = make_float2(m0, l0 * kUnscale);
        s_ml[warp][2 * t + 1] = make_float2(m1, l1 * kUnscale);
    }
    if (*abortp) {  // a wait ran out: what has been asked for lands within microseconds; do not use its place before
        if (lane == 0) flag(a.status, RIVER_E_TIMEOUT);
#pragma unroll 1
        for (int x = 0; x < 64; ++x) __nanosleep(4000);
    }
    __syncthreads();  // (nobody's blocks are under way: the rings become the warps' O)
#pragma unroll
    for (int d = 0; d < DH / 16; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_o[warp][2 * t + (e & 1)][16 * d + g + 8 * (e >> 1)] = o[d][e] * kUnscale;
    __syncthreads();
    // the warps' parts: a warp per head, lane = dims
    constexpr int E = DH / 32;
#pragma unroll 1
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
            for (int e = 0; e < E; e += 2) {
                const size_t at = (out + h) * DH + E * lane + e;
                if (direct) *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) + at) = pack_pair<T>(acc[e] * inv, acc[e + 1] * inv);
                else *reinterpret_cast<float2 *>(a.own_o + at) = make_float2(acc[e], acc[e + 1]);
            }
            if (!direct && lane == 0) a.own_ml[out + h] = make_float2(mm, ll);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) s_c[h][E * lane + e] = acc[e];
            if (lane == 0) s_cml[h] = make_float2(mm, ll);
        }
    }
    if (splits == 1) return leave();
    // the cluster's parts: every CTA finishes its share of the heads' dims
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
#pragma unroll 1
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
        if (direct) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) + out * DH + e) = pack_pair<T>(y0 * inv, y1 * inv);
        } else {
            *reinterpret_cast<float2 *>(a.own_o + out * DH + e) = make_float2(y0, y1);
            if (d == 0) a.own_ml[out + hd] = make_float2(top, sum);
        }
    }
    cluster.sync();  // (peers read this CTA's part)
    leave();
}

// Joining.  A part of a unit lies in the scratch as its CTA had it: its R rows' (the unit's tokens x heads) maxima and sums from ml[row] on, O from o[row * DH]
// on with four dims of all rows after four dims of all rows.  A warp joins 32 dims of up to eight rows: lane = row k = lane & 7, dims 4 (c + 4 i) .. + 3 of the
// 32, c = lane >> 3.  Bound by what each step waits for: code, the head, a unit's place, its parts' rows; 5 us for 64 rows of a group beside their own keys (one
// thread per dim of a row, O in the order of rows: 9), 10 for the cut units of a batch of prompts, two parts of 256 rows for most of 147 cuts.
__device__ __forceinline__ float pf_inf() { return CUDART_INF_F; }
__device__ __forceinline__ float pf_nan() { return CUDART_NAN_F; }
struct PfRows {
    float m = -pf_inf(), l = 0.f;
    float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    // U parts are under way together.  n parts (at most 32), lane j has the first row of part j among the scratch's (-1: nothing there); row r of R
    template <int U>
    __device__ __forceinline__ void add(const PrefixArgs &a, int64_t first, int n, int r, int R, int dh, int d4) {
#pragma unroll 1
        for (int j0 = 0; j0 < n; j0 += U) {
            float2 ml[U];
            float4 y[U][2];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int64_t row = __shfl_sync(0xffffffffu, first, (j0 + j) & 31);
                const bool there = j0 + j < n && row >= 0;
                const float4 *p = reinterpret_cast<const float4 *>(a.o + row * dh) + (int64_t)d4 * R + r;
                ml[j] = there ? __ldcg(a.ml + row + r) : make_float2(-pf_inf(), 0.f);
                y[j][0] = there ? __ldcg(p) : make_float4(0.f, 0.f, 0.f, 0.f);
                y[j][1] = there ? __ldcg(p + (int64_t)4 * R) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float most = m;
            bool odd = m != m;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                most = fmaxf(most, ml[j].x);
                odd = odd || ml[j].x != ml[j].x;
            }
            if (odd) most = pf_nan();
            const float base = most == -pf_inf() ? 0.f : most, old = m == -pf_inf() ? 0.f : ex2(m - base);
            m = most;
            l *= old;
#pragma unroll
            for (int i = 0; i < 2; ++i) { o[i].x *= old; o[i].y *= old; o[i].z *= old; o[i].w *= old; }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const float f = ml[j].x == -pf_inf() ? 0.f : ex2(ml[j].x - base);
                l += ml[j].y * f;
#pragma unroll
                for (int i = 0; i < 2; ++i) { o[i].x += y[j][i].x * f; o[i].y += y[j][i].y * f; o[i].z += y[j][i].z * f; o[i].w += y[j][i].w * f; }
            }
        }
    }
    // the parts of a unit that begins at weight x; first: of its first 32 CTAs; d4: this lane's first four dims of the row
    template <int U>
    __device__ __forceinline__ void add_unit(const PrefixArgs &a, int64_t share, int64_t x, const PfUnit &u, int kvh, int group, int64_t first, int r, int dh, int d4);
    template <class T>
    __device__ __forceinline__ void store(T *out) const {  // out: this lane's first dims
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<uint2 *>(out + 16 * i) = make_uint2(pack_pair<T>(o[i].x * inv, o[i].y * inv), pack_pair<T>(o[i].z * inv, o[i].w * inv));
    }
};
// CTAs that a unit's weight reaches into
__device__ __forceinline__ int pf_parts(int64_t share, int64_t x, const PfUnit &u) { return (int)pf_div(x + u.w - 1, share) - (int)pf_div(x, share) + 1; }
// the first row of the k-th one's part; -1: nothing there
static __device__ __noinline__ int64_t pf_part_row(const PfPlan &p, int64_t share, int64_t x, const PfUnit &u, int k, int kvh, int group) {
    const int c = (int)pf_div(x, share) + k;
    if (c >= kPfCtas || c * share >= x + u.w) return -1;
    const PfPart r = pf_part(p, share, x, u, c, kvh, group);
    return r.k1 > r.k0 ? r.row : -1;
}
template <int U>
__device__ __forceinline__ void PfRows::add_unit(const PrefixArgs &a, int64_t share, int64_t x, const PfUnit &u, int kvh, int group, int64_t first, int r, int dh, int d4) {
    const int n = min(pf_parts(share, x, u), kPfCtas);
#pragma unroll 1
    for (int k = 0; k < n; k += 32) {
        if (k) first = pf_part_row(a.p, share, x, u, k + (threadIdx.x & 31), kvh, group);
        add<U>(a, first, min(32, n - k), r, u.n * a.p.gq, dh, d4);
    }
}

// Rows with parts of a group's keys and of their own, a warp per token, up to eight heads of one KV head and 32 dims: 256 / DH tokens' tiles of eight heads per CTA.
// U parts are under way, CTAS CTAs share an SM: 8, 2 where all of them find a place at once, else 3, 4 - calls of 64 rows of one group, 256 of four, 2354 of six
// take 43, 164, 91 us by the first and 45, 160, 64 by the second.
template <class T, int DH, int U, int CTAS>
__global__ void __launch_bounds__(256, CTAS) prefix_join_kernel(const __grid_constant__ PrefixArgs a) {
    constexpr int Q = DH / 32, TILES = 8 / Q;  // warps of a tile; tiles of a CTA
    __shared__ int s_seq[TILES];
    const int gq = a.p.gq, span = 2 * pf_per(gq), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, S = a.c.n_seqs, rt = (gq + 7) / 8, tiles = a.c.Hkv * rt;
    const int64_t unit = (int64_t)blockIdx.x * TILES + warp / Q;
    const int first = (int)((int64_t)blockIdx.x * TILES / tiles), token = (int)(unit / tiles), tile = (int)(unit % tiles), kvh = tile / rt, g0 = tile % rt * 8;
    // the sequences of this CTA's tokens (single tokens' kernel has no place for those behind a sequence's max_q-th)
    if (threadIdx.x < TILES) s_seq[threadIdx.x] = -1;
    __syncthreads();
#pragma unroll 1
    for (int s = threadIdx.x; s < S; s += 256) {
        const int x = a.q_start[s], y = a.q_start[s + 1];
        if (x >= 0 && x < y && y <= a.p.n_tokens)
#pragma unroll 1
            for (int t = max(x, first); t < min(a.p.own ? y : min(y, x + a.max_q), first + TILES); ++t) s_seq[t - first] = s;
    }
    __syncthreads();
    const int seq = token < a.p.n_tokens ? s_seq[token - first] : -1, lead = seq < 0 ? -1 : a.lead[seq], shared = seq < 0 ? 0 : pf_shared(a.c, a.shared[seq]);
    const int heads = min(8, gq - g0), k = min(lane & 7, heads - 1), d4 = 8 * (warp % Q) + (lane >> 3);  // (lanes without a row repeat the last one)
    const bool grouped = shared > 0 && lead >= 0 && lead <= seq;
    const size_t row = (size_t)token * a.p.Hq + kvh * gq + g0 + k;
    pdl_wait();
    if (seq < 0) return;
    PfRows rows;
    if (!a.p.own) {
        const float2 ml = __ldcg(a.own_ml + row);
        rows.m = ml.x;
        rows.l = ml.y;
#pragma unroll
        for (int i = 0; i < 2; ++i) rows.o[i] = __ldcg(reinterpret_cast<const float4 *>(a.own_o + row * DH) + d4 + 4 * i);
    }
    const PfHead h = *a.head;
    const PfGroup g = grouped ? a.group[lead] : PfGroup{};
    if (grouped && pf_group_has(a.p, g.tok0, g.n, g.keys, token) && g.at >= 0 && g.at < h.all) {  // (else lead is no group's first sequence)
        const PfUnit u = pf_unit(pf_group_entry(g.tok0, g.n, lead, g.keys, span), (token - g.tok0) / span, span);
        const int64_t x = kvh * h.all + g.at + u.at;
        rows.add_unit<U>(a, h.share, x, u, kvh, 1, pf_part_row(a.p, h.share, x, u, lane, kvh, 1), (token - u.tok) * gq + g0 + k, DH, d4);
    }
    if (a.p.own) {
        const PfEntry e = pf_entry(a, S + seq, span);
        const PfUnit u = pf_unit(e, (token - e.tok0) / span, span);
        const int64_t x = kvh * h.all + a.own_at[seq] + u.at;
        rows.add_unit<U>(a, h.share, x, u, kvh, 0, pf_part_row(a.p, h.share, x, u, lane, kvh, 0), (token - u.tok) * gq + g0 + k, DH, d4);
    }
    if ((lane & 7) < heads) rows.store(static_cast<T *>(a.out) + row * DH + 4 * d4);
}
// Sequences' units that were cut: block (c, y) has the one that begins in CTA c's part, and a share of its rows.  Its parts are where those CTAs noted that
// they are: finding them by the arithmetic again, in cold code, took 4 to 8 us more.  (Two rows of a warp under way together gain nothing.)
constexpr int kJoinBlocks = 4;
template <class T, int DH>
__global__ void __launch_bounds__(256, 4) prefix_join_cut_kernel(const __grid_constant__ PrefixArgs a) {
    const int gq = a.p.gq, lane = threadIdx.x & 31, c = blockIdx.x;
    pdl_wait();
    const PfCut u = a.cut[c];
    auto head = [&](int k) { return c + k < kPfCtas && a.cut[c + k].head ? 2ll * (c + k) * a.p.slot_rows : -1; };  // first row of CTA c + k's part; -1: nothing there
    int64_t first = head(lane);
    if (u.n == 0) return;
    const int parts = u.last - c + 1;
    if (lane == 0) first = u.here ? (2ll * c + 1) * a.p.slot_rows : -1;
    bool any = __any_sync(0xffffffffu, lane < parts && first >= 0);  // (no: one CTA has every tile and the rows are written)
#pragma unroll 1
    for (int k = 32; k < parts; k += 32) any = any || __any_sync(0xffffffffu, k + lane < parts && head(k + lane) >= 0);
    if (!any) return;
    constexpr int Q = DH / 32;
    const int R = u.n * gq, w = blockIdx.y * 8 + (threadIdx.x >> 5), d4 = 8 * (w % Q) + (lane >> 3);
#pragma unroll 1
    for (int r0 = 8 * (w / Q); r0 < R; r0 += 64 * kJoinBlocks / Q) {
        const int r = min(r0 + (lane & 7), R - 1);  // (lanes without a row repeat the last one)
        PfRows rows;
#pragma unroll 1
        for (int k = 0; k < parts; k += 32) rows.add<2>(a, k ? head(k + lane) : first, min(32, parts - k), r, R, DH, d4);
        if (r0 + (lane & 7) < R) rows.store(static_cast<T *>(a.out) + ((size_t)(u.tok + r / gq) * a.p.Hq + u.kvh * gq + r % gq) * DH + 4 * d4);
    }
}

}  // namespace river

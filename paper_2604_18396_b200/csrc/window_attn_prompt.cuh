// Windowed attention of prompts on tcgen05 (sm_100a, internal).
//
// A CTA owns two tiles of 128 query rows - 128 / GQ consecutive tokens of one sequence x the GQ query heads of one KV head, token by
// token - and walks the blocks of 16 positions that some of its rows see (those of the sinks, then those of the windows' union), eight
// blocks = 128 keys at a time.  Both tiles use the same K and V:
//   S [128 x 128] = Q K^T     Q and K in shared memory, S in tensor memory
//   O [128 x DH] += P V       P (rounded to the inputs' type) in tensor memory over the place of S, V as it lies in the cache
//   warp 0        TMA: K and V pages, one 16 x 64 box per lane, three places for K, two for V
//   warp 1        tensor memory; one lane issues the MMAs: P V of a tile, S of its next keys, then the other tile's, so that the softmax of
//                 one tile runs under the MMAs of the other
//   warps 4..11   softmax, four per tile: thread = query row = TMEM lane; online, base 2, fp32; all 128 scores of a row in registers; O is
//                 rescaled only when a row's maximum has grown by more than 2^8 since it last was.  P goes out in two halves.
//
// What bounds it: a tile's chain - S, softmax, P V - of 2900 cycles for two query tiles, of which the tensor pipe needs 2240 (an MMA of 128 x 128 x 16
// takes 74 cycles with A in shared memory, 66 with A in tensor memory) and the special-function units 2048; and some 17000 cycles of a CTA's
// start and end.  8192 positions of the 8B class, window 4096: 405 us in a loop of seconds, 1.02 PFLOP/s of visible products, 340 to 365 in bursts (f16 2 %
// more, for the least number of a probability).
//
// P in 16 bits: its rounding weighs as much as the rounding of the result (2^-9 of sum p |v| against 2^-9 of the result in bf16, both
// random), and one product instead of two is half of the tensor pipe's work.  In f16 a probability below 2^-21 of the row's largest loses bits, and below
// 2^-31 it counts as 2^-31 (kWpBelow).
//
// Hidden positions: scores are replaced, not added to; V rows that no row of the CTA sees are set to zero in shared memory.  A row of V
// that some rows see and others do not is harmless as long as it is finite (0 x v); tiles that have such rows are looked through (f16: all
// of their rows), and where one holds an infinity or no number the CTA computes its rows again one by one (window_attn_row).  So it does for scores
// beyond kWpHuge.  That costs: 8192 positions, window 4096, 63 ms with one such value, 325 ms where all are, for 0.37.
#pragma once
#include "attn_prefill_tc.cuh"
#include "window_attn_step.cuh"

namespace river {

constexpr int kWpRows = 128, kWpKeys = 128, kWpThreads = 384, kWpMaxSplits = 4;
// Scores (log2) from which on the distance between a product and its rounded maximum, half a unit in the last place, is more than an exponent of P has
// room for: a CTA with such a row computes its rows one by one, which compares rounded scores with one another.
template <class T> constexpr float kWpHuge = std::is_same<T, __half>::value ? 8388608.f : 536870912.f;  // 2^23, 2^29
constexpr float kWpLazy = 8.f;  // growth of a row's maximum (log2) that O waits for before it is rescaled
// f16 ends at 2^-24 below and 2^16 above: there a row's m, which its probabilities 2^(s - m), their sum and O refer to, lies this far below its
// maximum, so that probabilities are as large as the type has room for beside the growth.
constexpr float kWpBelow = 7.f;

struct PromptArgs {
    WindowArgs w;
    int tiles;   // query tiles of a CTA: 1 or 2
    int splits;  // CTAs that share out the keys of a row, a cluster
    uint32_t polls = kWaitLimit;  // of a wait, before it gives up
    int mute = -1;                // self-test: the KV head whose first keys nobody asks for, so that waits run out
};

__device__ __forceinline__ void wp_ld32(uint32_t taddr, uint32_t (&r)[32]) {  // left under way (wp_ld_wait)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void wp_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Nothing that uses r moves above this point (the compiler does not know that r is filled only at the wait).
__device__ __forceinline__ void wp_pin(uint32_t (&r)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// One lane of the warp.  A warp runs its loop as a whole and only the tcgen05 instructions are one lane's: their operands live in
// uniform registers, and in a branch that the compiler must take for divergent each of them is carried there anew.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// Bounded wait.  Where it runs out the kernel goes on with whatever is there, every later wait ends at once, nothing more is loaded and no
// result of the CTA and its cluster is stored: nobody is left standing at a barrier.
__device__ __forceinline__ void wp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, uint32_t polls = kWaitLimit) {
    for (uint32_t it = 0; it < polls; ++it) {
        if (mbar_try_wait(bar, parity & 1u)) return;
        if (*abort_flag) return;
    }
    *abort_flag = 1;
}
// The same beside warps that may work for longer than that: they count `moved` up while they do, and a wait gives up after polls in which it stood still.  (Their
// work ends.  Looked at by every poll, a call of 43.5 us took 44.1.)
__device__ __forceinline__ void wp_wait(uint32_t bar, uint32_t parity, const volatile int *moved, volatile int *abort_flag, uint32_t polls) {
    int seen = 0;
    for (uint32_t it = 0; it < polls;) {
        if (mbar_try_wait(bar, parity & 1u)) return;
        if (*abort_flag) return;
        if (++it == polls) {
            const int now = *moved;
            if (now != seen) seen = now, it = 0;
        }
    }
    *abort_flag = 1;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// bits lo .. hi - 1 of a word, whatever the ends
__device__ __forceinline__ uint32_t bits_between(int lo, int hi) {
    const uint32_t below_hi = hi >= 32 ? 0xffffffffu : hi <= 0 ? 0u : (1u << hi) - 1u, below_lo = lo >= 32 ? 0xffffffffu : lo <= 0 ? 0u : (1u << lo) - 1u;
    return below_hi & ~below_lo;
}

// The sequence whose tiles hold slot x: sequence s has the slots from q_start[s] / per + s on, enough for its queries.
__device__ __forceinline__ int prompt_seq(const int32_t *q_start, int n_seqs, int per, int x) {
    int lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] / per <= x - mid) lo = mid; else hi = mid;
    }
    return lo;
}

// max of two pairs of f16, what is no number handed on
__device__ __forceinline__ uint32_t max2_f16_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// max of three that hands on what is no number
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Probabilities of 64 keys, w = 2^(s c - m) in pairs, and their sum on top of `sum`; in f16 each is at least that of `least`.  (The special-function units give 4 of them a cycle
// and quarter of an SM: 1024 of a tile's 1900 cycles.  A quarter, an eighth of them by a polynomial instead cost more than they saved,
// 160 -> 171, 167 us: with one warp of a query tile per quarter it is the length of its program that counts, not a unit's rate.)
template <class T>
__device__ __forceinline__ void wp_exps(const uint32_t (&a)[32], const uint32_t (&b)[32], uint64_t c2, uint64_t m2, uint32_t least, uint64_t &sum, uint32_t (&w)[32]) {
    uint64_t part[2] = {sum, 0ull};
    float p[32][2];
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const uint32_t *s = e < 16 ? a + 2 * e : b + 2 * e - 32;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(s[0]), __uint_as_float(s[1])), c2, m2), p[e][0], p[e][1]);
        p[e][0] = ex2(p[e][0]);
        p[e][1] = ex2(p[e][1]);
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        part[e & 1] = f2_add(part[e & 1], f2_pack(p[e][0], p[e][1]));
        w[e] = pack_pair<T>(p[e][0], p[e][1]);
        if constexpr (std::is_same<T, __half>::value) w[e] = max2_f16_nan(w[e], least);
    }
    sum = f2_add(part[0], part[1]);
}

// SPLIT: the key tiles of a row are shared out over a cluster, whose CTAs join their parts through distributed shared memory.
template <class T, int DH, bool SPLIT>
__global__ void __launch_bounds__(kWpThreads, 1) window_attn_prompt_kernel(const __grid_constant__ CUtensorMap tmap, const PromptArgs pa) {
    namespace cg = cooperative_groups;
    const WindowArgs &a = pa.w;
    constexpr int NB = DH / 64;                                          // blocks of 64 dims
    constexpr bool kHalf = std::is_same<T, __half>::value;
    constexpr uint32_t QB = kWpRows * 128, KB = kWpKeys * 128;           // bytes of one block of Q / of K or V
    constexpr uint32_t kO = 256;                                         // TMEM: tile q has S / P in columns 128 q .., O in 256 + DH q ..
    constexpr uint32_t kIdS = (1u << 4) | (sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) |
                              ((uint32_t)(kWpRows >> 4) << 24) | ((uint32_t)(kWpKeys >> 3) << 17);
    constexpr uint32_t kIdO = (kIdS & ~(0x3Fu << 17)) | ((uint32_t)(DH >> 3) << 17) | (1u << 16);  // (B of the second product: N-major)
    extern __shared__ uint8_t wp_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(wp_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *const sq = smem, *const sv = sq + 2 * NB * QB, *const sk = sv + 2 * NB * KB;  // [tile], [2 places of V], [3 of K] [NB][128 rows][128 bytes]
    float2 *const s_ml = reinterpret_cast<float2 *>(sk);  // SPLIT, at the end: a row's maximum and sum, for its cluster
    // K of the first tile there; V of tile j and K of tile j + 1 there (4, in turn); V of tile j and K before free (2); per query tile:
    // S done, P written (2), O done; Q there
    __shared__ uint64_t bars[16];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_no_page, s_poison, s_missing;
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int gq = a.Hq / a.c.Hkv, per = kWpRows / gq;  // tokens of a tile
    // heavy tiles, those behind a long history, first
    const int splits = SPLIT ? pa.splits : 1, unit = blockIdx.x / splits, kvh = unit % a.c.Hkv, slot = gridDim.x / splits / a.c.Hkv - 1 - unit / a.c.Hkv;
    const int seq = prompt_seq(a.q_start, a.c.n_seqs, per * pa.tiles, slot);
    const int first = a.q_start[seq], end = a.q_start[seq + 1];  // (compared before they are subtracted: any ints may stand there)
    const int n = first < 0 || end < first || end > a.n_tokens ? 0 : end - first, at = n == 0 ? 0 : (slot - (first / (per * pa.tiles) + seq)) * per * pa.tiles;
    if (blockIdx.x == 0)
        for (int s = tid; s < a.c.n_seqs; s += kWpThreads) {
            const int x = a.q_start[s], y = a.q_start[s + 1];
            if (x < 0 || y < x || y > a.n_tokens || y - x > a.max_q) flag(a.status, RIVER_E_BADARG);
        }
    if (at < 0 || at >= n) return;
    const int n_tok = min(n - at, per * pa.tiles), tok0 = first + at, pos0 = window_len(a, a.c.lens[seq]) - n + at, last_pos = pos0 + n_tok - 1;
    const int nq = n_tok > per ? 2 : 1;

    const uint32_t b_first = smem_u32(&bars[0]), b_full = b_first + 8, b_free = b_full + 32, b_s = b_free + 16, b_p = b_s + 16, b_o = b_p + 32, b_q = b_o + 16;
    volatile int *abortp = &s_abort;
    if (tid == 0) {
        s_abort = s_no_page = s_poison = s_missing = 0;
        for (int i = 0; i < 16; ++i) mbar_init(smem_u32(&bars[i]), i >= 9 && i < 13 ? 4 : i == 15 ? 8 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        tc_alloc(smem_u32(&s_tmem), 512u);
        tc_fence_before();
    }
    // blocks of 16 positions: n_sb of the sinks, then wb0 .. last_pos / 16; a column is a place on that list, of position column
    // (sinks) or column + shift
    const int low0 = window_low(pos0, a.window), wb0 = low0 >> 4, n_sb = min((min(a.sinks, low0) + 15) >> 4, wb0), shift = 16 * (wb0 - n_sb);
    const int nb_all = last_pos < 0 ? 0 : n_sb + (last_pos >> 4) - wb0 + 1, n_all = (nb_all + 7) / 8;
    // this CTA's tiles of 128 columns: t0 .. t0 + n_kt - 1, of its blocks 8 t0 .. nb - 1
    const int split = SPLIT ? blockIdx.x % splits : 0, t0 = SPLIT ? n_all * split / splits : 0, n_kt = SPLIT ? n_all * (split + 1) / splits - t0 : n_all;
    const int nb = SPLIT ? min(nb_all, 8 * (t0 + n_kt)) : nb_all;

    const int32_t *const tbl = a.c.table + (size_t)seq * a.c.max_pages;
    auto block_of = [&](int u) { return u < n_sb ? u : wb0 + u - n_sb; };
    auto page_of = [&](int u) {  // of the u-th block; -1: none
        const int col = block_of(u) >> (a.c.ps_log2 - 4), page = u < nb && col < a.c.max_pages ? tbl[col] : -1;
        return page < a.c.n_pages ? max(page, -1) : -1;
    };

    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(s_tmem);

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0) {
            const int blk = lane / NB, half = lane % NB;
            int ahead = blk < 8 ? page_of(8 * t0 + blk) : -1, place = 0;
            auto load = [&](uint8_t *dst, int page, int j, int v, uint32_t bar) {
                const int row = ((page * 2 * a.c.Hkv + kvh + v * a.c.Hkv) << a.c.ps_log2) + ((block_of(8 * (t0 + j) + blk) << 4) & ((1 << a.c.ps_log2) - 1));
                if (page >= 0) tma_load_2d(smem_u32(dst) + half * KB + blk * 2048, &tmap, 64 * half, row, bar);
            };
            // K of tile j + 1 comes together with V of tile j
            int page = -1;  // of tile j
            uint32_t bytes = 0;
            for (int j = pa.mute == kvh && t0 == 0 ? n_kt : -1; j < n_kt; ++j) {
                const int next = ahead;  // of tile j + 1
                ahead = blk < 8 ? page_of(8 * (t0 + j + 2) + blk) : -1;  // (under way while this tile waits for its place)
                if (blk < 8 && 8 * (t0 + j + 1) + blk < nb && next < 0) s_no_page = 1;
                const uint32_t k_bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, next >= 0)) * 2048u, bar = j < 0 ? b_first : b_full + 8 * (j & 3);
                if (j >= 2) wp_wait(b_free + 8 * (j & 1), (j >> 1) - 1, abortp, pa.polls);
                if (__any_sync(0xffffffffu, *abortp)) break;
                if (lane == 0) mbar_expect_tx(bar, bytes + k_bytes);
                __syncwarp();
                load(sk + place * NB * KB, next, j + 1, 0, bar);
                if (j >= 0) load(sv + (j & 1) * NB * KB, page, j, 1, bar);
                page = next;
                bytes = k_bytes;
                place = place == 2 ? 0 : place + 1;
            }
        } else if (warp == 1) {
            const uint64_t dq = tc_smem_desc(smem_u32(sq)), dk = tc_smem_desc(smem_u32(sk)), dv = pt_desc_n(smem_u32(sv), KB);
            const int n_t = uniform(n_kt), n_q = uniform(nq);
            const bool leader = elect_one();
            auto scores = [&](int q, uint64_t k_desc) {
#pragma unroll
                for (int k = 0; k < DH / 16; ++k)
                    tc_mma(tmem + 128u * q, dq + (q * NB + (k >> 2)) * (QB >> 4) + 2 * (k & 3), k_desc + (k >> 2) * (KB >> 4) + 2 * (k & 3), kIdS, k ? 1u : 0u);
                tc_commit(b_s + 8 * q);
            };
            if (n_t > 0) {
                wp_wait(b_q, 0, abortp, pa.polls);
                wp_wait(b_first, 0, abortp, pa.polls);
                tc_fence_after();
                if (leader) {
                    scores(0, dk);
                    if (n_q == 2) scores(1, dk);
                }
            }
            int place = 0;
            for (int j = 0; j < n_t; ++j) {
                place = place == 2 ? 0 : place + 1;  // of K of the next tile
                const uint64_t v = dv + (j & 1) * (NB * KB >> 4), k_desc = dk + place * (NB * KB >> 4);
                wp_wait(b_full + 8 * (j & 3), j >> 2, abortp, pa.polls);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (q == 1 && n_q == 1) break;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // half of the keys
                        wp_wait(b_p + 8 * (2 * q + h), j, abortp, pa.polls);
                        tc_fence_after();
                        if (leader) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)  // 16 keys: 8 columns of P, 2048 bytes of V
                                tc_mma_ts(tmem + kO + (uint32_t)DH * q, tmem + 128u * q + 32 * h + 8 * k, v + (4 * h + k) * (2048 >> 4), kIdO, (j | h | k) ? 1u : 0u);
                            if (h == 1) {
                                if (q == n_q - 1) tc_commit(b_free + 8 * (j & 1));
                                if (j + 1 < n_t) scores(q, k_desc);
                                else tc_commit(b_o + 8 * q);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        {  // ---- Q rows in the operand's swizzled order (a negative scale turns their signs); rows that are none are zero
            const uint32_t turn = a.scale_log2 < 0.f ? 0x80008000u : 0u;
            constexpr int C8 = DH / 8, U = C8;  // 16-byte chunks of a row; all of a thread's are under way together
            const int u0 = tid - 128, c8 = u0 % C8, inv_gq = 65536 / gq + 1;  // (r * inv_gq >> 16 = r / gq for r < 128)
            const T *src = static_cast<const T *>(a.q) + tok0 * a.q_tok + kvh * gq * a.q_head + 8 * c8;
            uint4 x[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int rr = u0 / C8 + i * (256 / C8), r = rr % kWpRows, pp = r * inv_gq >> 16, p = rr / kWpRows * per + pp, g = r - pp * gq;
                x[i] = make_uint4(0u, 0u, 0u, 0u);
                if (pp < per && p < n_tok) x[i] = *reinterpret_cast<const uint4 *>(src + p * a.q_tok + g * a.q_head);
            }
            bool missing = false;
            for (int u = 8 * t0 + u0; u < nb; u += 256) missing = missing || page_of(u) < 0;
            if (missing) s_missing = 1;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int rr = u0 / C8 + i * (256 / C8), r = rr % kWpRows;
                x[i].x ^= turn; x[i].y ^= turn; x[i].z ^= turn; x[i].w ^= turn;
                *reinterpret_cast<uint4 *>(sq + rr / kWpRows * NB * QB + (c8 >> 3) * QB + r * 128 + (((c8 & 7) ^ (r & 7)) * 16)) = x[i];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q);
            asm volatile("bar.sync 1, 256;" ::: "memory");  // (s_missing)
        }
        const int q = (warp - 4) >> 2, r = 32 * (warp & 3) + lane, p = q * per + r / gq;
        float m = -CUDART_INF_F, l = 0.f;
        if (q < nq) {
            const int pos = pos0 + min(p, n_tok - 1);
            const int c_sink = min(a.sinks, max(pos + 1, 0)), c_lo = window_low(pos, a.window) - shift, c_hi = pos + 1 - shift;  // columns seen: [0, c_sink), [c_lo, c_hi)
            // over all rows of the CTA
            const int all_lo = window_low(last_pos, a.window) - shift, all_hi = pos0 + 1 - shift, any_lo = low0 - shift, any_hi = last_pos + 1 - shift;
            const int all_sink = min(a.sinks, max(pos0 + 1, 0)), any_sink = min(a.sinks, last_pos + 1);
            const uint32_t quarter = (uint32_t)(32 * (warp & 3)) << 16, t_s = tmem + 128u * q + quarter, t_o = tmem + kO + (uint32_t)DH * q + quarter;
            const float c = fmaxf(fabsf(a.scale_log2), 1e-30f);  // (a scale of 0: every score 0, hidden ones -inf still)
            const bool missing = s_missing != 0;
            auto huge = [&] { if (fabsf(m) > kWpHuge<T> && m != -CUDART_INF_F) s_poison = 1; };
            for (int j = 0; j < n_kt; ++j) {
                const int c0 = 128 * (t0 + j);
                uint32_t valid = 0xffu;  // blocks that are there
                bool part = !(c0 >= all_lo && c0 + 128 <= all_hi) && !(c0 + 128 <= all_sink);
                if (missing) {
#pragma unroll 1
                    for (int i = 0; i < 8; ++i)
                        if (8 * (t0 + j) + i < nb && page_of(8 * (t0 + j) + i) < 0) valid &= ~(1u << i);
                    part = part || valid != 0xffu;
                }
                if (part && q == 0) {  // thread = V row: those that nobody sees become zero, the others are looked through
                    wp_wait(b_full + 8 * (j & 3), j >> 2, abortp, pa.polls);
                    const int cc = c0 + r;
                    uint8_t *row = sv + (j & 1) * NB * KB + r * 128;
                    if (!kHalf && (valid >> (r >> 4) & 1u) && (cc < all_sink || (cc >= all_lo && cc < all_hi))) {
                        // (seen by every row: whatever it is, it belongs in every result)
                    } else if ((valid >> (r >> 4) & 1u) && (cc < any_sink || (cc >= any_lo && cc < any_hi))) {
                        // an exponent of ones (what is no number) and one more carries into the sign's place
                        constexpr uint32_t E = std::is_same<T, __nv_bfloat16>::value ? 0x7f807f80u : 0x7c007c00u, ONE = E & ~(E << 1);
                        uint32_t odd = 0u;
#pragma unroll
                        for (int i = 0; i < DH / 8; ++i) {
                            const uint4 y = *reinterpret_cast<const uint4 *>(row + (i >> 3) * KB + (((i & 7) ^ (r & 7)) * 16));
                            odd |= ((y.x & E) + ONE) | ((y.y & E) + ONE) | ((y.z & E) + ONE) | ((y.w & E) + ONE);
                        }
                        if (odd & 0x80008000u) s_poison = 1;
                    } else {
#pragma unroll
                        for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<uint4 *>(row + (i >> 3) * KB + (((i & 7) ^ (r & 7)) * 16)) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                wp_wait(b_s + 8 * q, j, abortp, pa.polls);
                __syncwarp();
                tc_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) wp_ld32(t_s + 32 * i, s[i]);
                wp_ld_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i) wp_pin(s[i]);
                if (part) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int cc = c0 + 32 * i;
                        const uint32_t there = (valid >> (2 * i) & 1u ? 0xffffu : 0u) | (valid >> (2 * i + 1) & 1u ? 0xffff0000u : 0u);
                        const uint32_t see = (bits_between(0, c_sink - cc) | bits_between(c_lo - cc, c_hi - cc)) & there;
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[i][e] = see >> e & 1u ? s[i][e] : 0xff800000u;  // -inf
                    }
                }
                // The first half is made with the maximum as it stood; only where the tile's own maximum, found meanwhile, has grown too
                // far past it (a first tile, a rare later one) it is made again.
                uint64_t sum;
                uint32_t w[32];
                // A probability that f16 has no number for would make 0 x inf of an infinite value: where every row sees every key it counts as 2^-24
                // (2^-31 of the row's largest); tiles in parts are looked through.
                const uint32_t least = part ? 0u : 0x00010001u;
                const uint64_t c2 = f2_pack(c, c);
                if (j == 0) {
                    float x[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) x[(e >> 1) & 3] = max3_nan(x[(e >> 1) & 3], __uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1]));
                    const float mx = max3_nan(max3_nan(x[0], x[1], x[2]), x[3], x[3]) * c;
                    m = mx < CUDART_INF_F ? (kHalf ? mx - kWpBelow : mx) : CUDART_NAN_F;
                    huge();
                }
                while (true) {
                    sum = 0ull;
                    const float base = m == -CUDART_INF_F ? 0.f : m;
                    float x[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) x[(e >> 1) & 3] = max3_nan(x[(e >> 1) & 3], __uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1]));
                    const float mx = max3_nan(max3_nan(x[0], x[1], x[2]), x[3], x[3]) * c;
                    wp_exps<T>(s[0], s[1], c2, f2_pack(-base, -base), least, sum, w);
                    bool grow;
                    float corr;
                    if constexpr (kHalf) {  // (by the difference, which is exact where the two are near: no rounding of a large m makes P infinite)
                        grow = !(mx - fmaxf(m, -3e38f) <= kWpLazy + kWpBelow) && !(m != m);
                        corr = grow ? ex2(m - (mx - kWpBelow)) : 1.f;
                    } else {
                        grow = !(mx <= m + kWpLazy) && !(m != m);  // (a maximum that is no number stays)
                        corr = grow ? ex2(m - mx) : 1.f;
                    }
                    if (!__any_sync(0xffffffffu, grow)) break;
                    if (grow) m = mx < CUDART_INF_F ? (kHalf ? mx - kWpBelow : mx) : CUDART_NAN_F;  // (inf - inf, as the formula has it)
                    huge();
                    l *= corr;
                    if (j > 0) {  // (the MMAs that wrote O are complete: S of these keys was issued behind them)
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
                auto hand_over = [&](int h) {
                    tc_st32(t_s + 32 * h, w);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_p + 8 * (2 * q + h));
                };
                hand_over(0);
                wp_pin(s[2]);  // (no probability of the second half before the first is handed over)
                wp_pin(s[3]);
                {
                    const float base = m == -CUDART_INF_F ? 0.f : m;
                    wp_exps<T>(s[2], s[3], c2, f2_pack(-base, -base), least, sum, w);
                }
                hand_over(1);
                float l0, l1;
                f2_unpack(sum, l0, l1);
                l += l0 + l1;
            }
            if (n_kt > 0) wp_wait(b_o + 8 * q, 0, abortp, pa.polls);
            __syncwarp();
            tc_fence_after();
            if constexpr (!SPLIT) {
                const bool none = m == -CUDART_INF_F;  // (no key seen: O may be 0 x whatever)
                const float inv = none ? 0.f : 1.f / l;
                uint4 *const mine = reinterpret_cast<uint4 *>(sq + q * NB * QB);  // (rows through the place of this tile's Q: whole lines of them go out)
                constexpr int C8 = DH / 8;
#pragma unroll 1
                for (int d = 0; d < DH; d += 32) {
                    uint32_t o[32], w[16];
                    if (n_kt > 0) {
                        wp_ld32(t_o + d, o);
                        wp_ld_wait();
                        wp_pin(o);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = none ? 0u : pack_pair<T>(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
#pragma unroll
                    for (int e = 0; e < 4; ++e) mine[r * C8 + ((d / 8 + e) ^ (r & (C8 - 1)))] = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                }
                __syncwarp();
                const int lr = lane / C8, lc = lane % C8, inv_gq = 65536 / gq + 1;
                if (!*abortp)
#pragma unroll 4
                    for (int i = 0; i < 32; i += 32 / C8) {
                        const int rr = 32 * (warp & 3) + i + lr, pp = rr * inv_gq >> 16, t = q * per + pp;
                        if (pp < per && t < n_tok)
                            *reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + ((size_t)(tok0 + t) * a.Hq + kvh * gq + rr - pp * gq) * DH + 8 * lc) = mine[rr * C8 + (lc ^ (rr & (C8 - 1)))];
                    }
                tc_fence_before();
            }
        }
        if constexpr (SPLIT) {
            asm volatile("bar.sync 1, 256;" ::: "memory");  // (both tiles' MMAs are complete: the places of Q and V are free, and those of K)
            if (q < nq) {
                s_ml[q * kWpRows + r] = make_float2(m, l);
                float4 *const mine = reinterpret_cast<float4 *>(smem) + (q * kWpRows + r) * (DH / 4);
                if (n_kt > 0)
#pragma unroll 1
                    for (int d = 0; d < DH; d += 32) {
                        uint32_t o[32];
                        wp_ld32(tmem + kO + (uint32_t)DH * q + ((uint32_t)(32 * (warp & 3)) << 16) + d, o);
                        wp_ld_wait();
                        wp_pin(o);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            mine[(d / 4 + e) ^ (r & (DH / 4 - 1))] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    }
            }
            tc_fence_before();
        }
    }
    __syncwarp();
    if (*abortp) {  // a wait ran out: what this CTA has asked for lands within microseconds; do not leave before
        for (int i = 0; i < 64; ++i) __nanosleep(4000);
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tc_dealloc(tmem, 512u);
    }
    bool gave_up = *abortp != 0;
    if (tid == 0 && (gave_up || s_no_page)) flag(a.status, gave_up ? RIVER_E_TIMEOUT : RIVER_E_BADARG);
    if constexpr (SPLIT) {
        // ---- the cluster's parts of a row, a row (dh 64: two) per warp: every CTA finishes its share of the rows.  (Not warps 0 .. 3, which have
        // few registers left.)
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        for (int k = 0; k < splits; ++k) gave_up = gave_up || *cluster.map_shared_rank(&s_abort, k) != 0;
        constexpr int L = DH / 4;  // lanes of a row
        const int rows = nq * kWpRows, mine = (rows + splits - 1) / splits;
        for (int i = (warp - 4) * (32 / L) + lane / L; warp >= 4 && !gave_up && i < mine; i += 256 / L) {
            const int rr = split * mine + i, r = rr % kWpRows, t = rr / kWpRows * per + r / gq;
            if (rr >= rows || r >= per * gq || t >= n_tok) continue;
            const int chunk = lane % L;
            float2 ml[kWpMaxSplits];
            float4 o[kWpMaxSplits];
#pragma unroll
            for (int k = 0; k < kWpMaxSplits; ++k) {
                ml[k] = make_float2(-CUDART_INF_F, 0.f);
                if (k >= splits) continue;
                ml[k] = *cluster.map_shared_rank(&s_ml[rr], k);
                o[k] = *cluster.map_shared_rank(reinterpret_cast<const float4 *>(smem) + rr * (DH / 4) + (chunk ^ (r & (DH / 4 - 1))), k);
            }
            float top = -CUDART_INF_F, sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kWpMaxSplits; ++k) top = fmaxf(top, ml[k].x);
            const float base = top == -CUDART_INF_F ? 0.f : top;
#pragma unroll
            for (int k = 0; k < kWpMaxSplits; ++k) {
                if (ml[k].x == -CUDART_INF_F) continue;  // (that CTA has no key of this row: its O may be anything)
                const float f = ex2(ml[k].x - base);
                sum += ml[k].y * f;
                y.x += o[k].x * f; y.y += o[k].y * f; y.z += o[k].z * f; y.w += o[k].w * f;
            }
            const float inv = top == -CUDART_INF_F && sum == 0.f ? 0.f : 1.f / sum;
            *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + ((size_t)(tok0 + t) * a.Hq + kvh * gq + r % gq) * DH + 4 * chunk) =
                make_uint2(pack_pair<T>(y.x * inv, y.y * inv), pack_pair<T>(y.z * inv, y.w * inv));
        }
        cluster.sync();  // (peers read this CTA's part; and no row is written any more)
    }
    if (s_poison && warp >= 4 && !gave_up)
#pragma unroll 1
        for (int r = warp - 4; r < n_tok * gq; r += 8) window_attn_row<T, DH>(a, tok0 + r / gq, kvh * gq + r % gq, seq, pos0 + r / gq);
}

// (the head dim of 64 asks for as much as 128 does: no CTA that wants tensor memory shares an SM with one that holds all of it)
inline size_t window_attn_prompt_smem() { return 1024 + 7 * 2 * 128 * 128; }

// Query tiles of a CTA and CTAs of a cluster, by an estimate of the time in us: a CTA takes 8 for its start and end, 1.4 (one query
// tile) or 1.7 (two) for each of its key tiles, and 4 for the joining where the keys are split; up to one CTA per SM at a time.  One
// prompt, window 1024, 8B-class heads, 64 new tokens: 21 us with whole rows, 17 over four CTAs; 4096 positions of 8 heads without groups 111
// us with one query tile to a CTA, 74 with two.
inline void prompt_shape(PromptArgs &pa, int num_sms, double &best_t) {
    const WindowArgs &a = pa.w;
    const int per = kWpRows / (a.Hq / a.c.Hkv);
    best_t = 1e300;
    for (int tiles = 2; tiles >= 1; --tiles)
        for (int splits = 1; splits <= kWpMaxSplits; splits *= 2) {
            const int span = per * tiles;
            const double keys = (double)std::min<int64_t>((int64_t)a.c.max_pages << a.c.ps_log2, (int64_t)a.window + span + a.sinks), kt = std::ceil(keys / 128.0 + 0.5);
            const double parts = a.c.n_seqs == 1 ? std::ceil((double)a.n_tokens / span) : std::max((double)a.c.n_seqs, (double)a.n_tokens / span + 0.5 * a.c.n_seqs);
            const double rounds = parts * a.c.Hkv * splits / num_sms;
            const double one = 8.0 + std::ceil(kt / splits) * (tiles == 1 ? 1.4 : 1.7) + (splits > 1 ? 4.0 : 0.0);
            const double t = one * (rounds <= 1.0 ? 1.0 : rounds <= 2.0 ? 2.0 : rounds + 0.3);
            if (t < 0.97 * best_t) {
                best_t = t;
                pa.tiles = tiles;
                pa.splits = splits;
            }
        }
}

}  // namespace river

// Deciding which page goes where: prefix sums over sequences and page ids by one cluster of CTAs (internal).
#pragma once
#include <algorithm>

#include <cooperative_groups.h>

#include "paged_common.cuh"

namespace river {

namespace cg = cooperative_groups;

constexpr int kPgThreads = 1024;
constexpr int kPgSeqs = 8192;    // sequences whose prefix sums are held in shared memory
constexpr int kPgSeqInts = 5;    // of a reordering, per sequence in (dynamic) shared memory
constexpr int kPgCtas = 8;       // of the deciding cluster (a portable size)
constexpr int kPgRuns = 4;       // of page ids per warp, where free ones are looked for

// Shared memory of a deciding CTA; `count` is read and the first one's `odd` written by the other CTAs of the cluster.
struct PagesScan {
    int part[33], count[2];
    int runs[kPgRuns * 32 * 2 * kPgCtas];  // free ids per run, written by all CTAs of the cluster, then how many there are before
    int bad, full;  // what every CTA finds for itself: a sequence or length out of range, a row too long
    int odd;        // a page out of range: the first CTA's tells, behind a barrier of the cluster
    unsigned long long wanted;  // of all sequences, where 32 bits may not hold it
};
struct PagesShared : PagesScan {
    int prefix[kPgSeqs];
};

// Exclusive prefix sum over the CTA's threads (`part`: 33 ints); `total` gets the sum.  Ends with a barrier behind every read.
__device__ __forceinline__ int cta_scan(int x, int *part, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int p = part[lane], i = p;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, i, o);
            if (lane >= o) i += y;
        }
        part[lane] = i - p;
        if (lane == 31) part[32] = i;
    }
    __syncthreads();
    const int before = part[warp] + inc - x;
    total = part[32];
    __syncthreads();
    return before;
}

// s[0 .. n): counts in, their exclusive prefix sums out; returns the sum.
__device__ inline int scan_shared(int *s, int n, int *part) {
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += kPgThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const int before = cta_scan(i < n ? s[i] : 0, part, total);
        if (i < n) s[i] = base + before;
        base += total;
    }
    __syncthreads();
    return base;
}

// The page ids of a thread: a range per CTA, in it a run of whole fours per thread.
struct Run {
    int lo, hi;
    __device__ __forceinline__ Run(int n, int rank, int ctas) {
        const int per = (int)(((int64_t)n + (int64_t)ctas * kPgThreads - 1) / ((int64_t)ctas * kPgThreads) + 3) & ~3;
        lo = (int)min((int64_t)n, ((int64_t)rank * kPgThreads + threadIdx.x) * per);
        hi = min(n, lo + per);
    }
    // f(id, refs of it) in ascending order
    template <class F>
    __device__ __forceinline__ void each(const int32_t *refs, F f) const {
        if ((reinterpret_cast<uintptr_t>(refs) & 15) == 0) {
            for (int p = lo; p + 4 <= hi; p += 4) {
                const int4 r = __ldcg(reinterpret_cast<const int4 *>(refs + p));
                f(p, r.x); f(p + 1, r.y); f(p + 2, r.z); f(p + 3, r.w);
            }
            for (int p = lo + ((hi - lo) & ~3); p < hi; ++p) f(p, __ldcg(refs + p));
        } else {
            for (int p = lo; p < hi; ++p) f(p, __ldcg(refs + p));
        }
    }
};
// Of the ids that `mine` counts per thread: how many there are before this thread's, and (all) in the whole cluster.  All threads.
__device__ __forceinline__ int cluster_scan(int mine, PagesScan &s, cg::cluster_group &cluster, int &all) {
    const int rank = cluster.block_rank(), ctas = cluster.num_blocks();
    int total;
    int before = cta_scan(mine, s.part, total);
    all = total;
    if (ctas == 1) return before;
    if (threadIdx.x == 0) s.count[0] = total;
    cluster.sync();
    all = 0;
    for (int c = 0; c < ctas; ++c) {
        const int x = *cluster.map_shared_rank(&s.count[0], c);
        if (c < rank) before += x;
        all += x;
    }
    cluster.sync();  // (counts have been read)
    return before;
}

// give(k, id) for the `want` lowest ids with refs 0, ascending, if there are as many; returns whether there are.  All threads of the cluster.
// A warp has kPgRuns runs of ids, and neighbouring runs are different CTAs': the lowest ids, which are given, are everybody's.
template <class F>
__device__ inline bool lowest_free(const int32_t *refs, int n_pages, int want, PagesScan &s, cg::cluster_group &cluster, F give) {
    constexpr int U = 4;  // times 32 ids under way
    const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = kPgRuns * 32 * ctas;
    const int64_t per = ((int64_t)n_pages + 32 * (int64_t)n - 1) / (32 * n) * 32;
    auto run_of = [&](int t) { return (32 * t + warp) * ctas + rank; };
    // f(id, lanes whose ids are free) over a run until it answers no
    auto each = [&](int run, auto f) {
        const int64_t lo = min((int64_t)n_pages, run * per), hi = min((int64_t)n_pages, lo + per);
        for (int64_t p0 = lo; p0 < hi; p0 += 32 * U) {
            int r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t p = p0 + 32 * u + lane;
                r[u] = p < hi ? __ldcg(refs + p) : 1;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (!f((int)(p0 + 32 * u + lane), __ballot_sync(0xffffffffu, r[u] == 0))) return;
        }
    };
#pragma unroll
    for (int t = 0; t < kPgRuns; ++t) {
        int mine = 0;
        each(run_of(t), [&](int, unsigned free) { mine += __popc(free); return true; });
        if (lane < ctas) *cluster.map_shared_rank(&s.runs[run_of(t)], lane) = mine;
    }
    cluster.sync();
    // free ids before each run
    int all = 0;
    for (int i0 = 0; i0 < n; i0 += kPgThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const int before = cta_scan(i < n ? s.runs[i] : 0, s.part, total);
        if (i < n) s.runs[i] = all + before;
        all += total;
    }
    __syncthreads();
    if (all < want) return false;
    for (int t = 0; t < kPgRuns; ++t) {
        int k = s.runs[run_of(t)];
        if (k < want)
            each(run_of(t), [&](int p, unsigned free) {
                const int rank_of = k + __popc(free & ((1u << lane) - 1u));
                if ((free >> lane & 1u) && rank_of < want) give(rank_of, p);
                k += __popc(free);
                return k < want;
            });
    }
    return true;
}
// the last i < n with prefix[i] <= k (prefix[0] = 0): whose want number k is
__device__ __forceinline__ int owner_of(const int *prefix, int n, int k) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}
// n ints, by all threads of the cluster
__device__ __forceinline__ void copy_ints(int32_t *to, const int32_t *from, size_t n, int thread, int threads) {
    if (((reinterpret_cast<uintptr_t>(to) | reinterpret_cast<uintptr_t>(from)) & 15) == 0) {
        int4 *t = reinterpret_cast<int4 *>(to);
        const int4 *f = reinterpret_cast<const int4 *>(from);
        size_t i = thread;
        for (; i + 3 * (size_t)threads < n / 4; i += 4 * (size_t)threads) {
            int4 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = f[i + e * (size_t)threads];
#pragma unroll
            for (int e = 0; e < 4; ++e) t[i + e * (size_t)threads] = v[e];
        }
        for (; i < n / 4; i += threads) t[i] = f[i];
        for (i = n / 4 * 4 + thread; i < n; i += threads) to[i] = from[i];
    } else {
        for (size_t i = thread; i < n; i += threads) to[i] = from[i];
    }
}

// work: table entries and page ids.  A few thousand are one CTA's; from 2^18 on twice the portable cluster pays (256 sequences of 2048
// pages, 65536 ids: 24 -> 17 us).
// beside: it may start before the kernel before it has ended.
template <class A>
int launch_deciding(void (*kernel)(A), const A &a, size_t work, size_t smem, cudaStream_t st, bool beside = false) {
    const unsigned ctas = work <= 4 * kPgThreads ? 1 : work < (1u << 18) ? kPgCtas : 2 * kPgCtas;
    if (ctas > 8 && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return RIVER_E_DEVICE;
    // the limit belongs to the kernel, not to the call: whoever sets it sets the same one, or a launch of another thread could fail by it
    constexpr int most = kPgSeqInts * sizeof(int) * kPgSeqs;
    if (smem > (32u << 10) && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most))) return RIVER_E_DEVICE;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPgThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = beside ? 2 : ctas > 1 ? 1 : 0;
    return cuda_rc(cudaLaunchKernelEx(&cfg, kernel, a));
}

}  // namespace river

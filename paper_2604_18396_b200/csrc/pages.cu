// river_pages_advance, river_pages_reorder, river_pages_compact: the pages of a paged cache, kept on the device.
//
// Which page goes where is decided by one cluster of CTAs: a few prefix sums over sequences (every CTA for itself, in shared memory)
// and over page ids (a range of ids per CTA, the ranges' counts through distributed shared memory).  Free pages are those with refs
// 0 after what the call gives back; the k-th page that is wanted, in order of (sequence, position), receives the k-th free id.  The
// values then move in a kernel of their own, over all SMs, that reads the list of copies.
#include <algorithm>

#include <cooperative_groups.h>

#include "paged_common.cuh"

namespace river {
namespace {

namespace cg = cooperative_groups;

constexpr int kPgThreads = 1024;
constexpr int kPgSeqs = 8192;    // sequences whose prefix sums are held in shared memory
constexpr int kPgSeqInts = 5;    // of a reordering, per sequence in (dynamic) shared memory
constexpr int kPgCtas = 8;       // of the deciding cluster (a portable size)

struct PagesArgs {
    Paged c;
    const int32_t *refs, *n_new, *parents;
    int window, sinks;
    int32_t *table_out, *lens_out, *refs_out, *list, *status;  // list: of copies or moves
    int32_t *remap, *n_used;
    int copy_here;  // the deciding cluster copies as well
};

// Shared memory of a deciding CTA; `count` is read and the first one's `odd` written by the other CTAs of the cluster.
struct PagesScan {
    int part[33], count[2];
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
__device__ int scan_shared(int *s, int n, int *part) {
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
template <class F>
__device__ bool lowest_free(const int32_t *refs, int n_pages, int want, PagesScan &s, cg::cluster_group &cluster, F give) {
    const Run run(n_pages, cluster.block_rank(), cluster.num_blocks());
    int mine = 0, all;
    run.each(refs, [&](int, int r) { mine += r == 0; });
    int k = cluster_scan(mine, s, cluster, all);
    if (all < want) return false;
    if (mine > 0 && k < want)
        run.each(refs, [&](int p, int r) {
            if (r == 0) {
                if (k < want) give(k, p);
                ++k;
            }
        });
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

// One head's values of a page, of one block, by a warp: its filled positions are consecutive, and 4 KB are under way.
__device__ __forceinline__ void copy_head(const Paged &c, int l, int head, int src, int dst, int positions) {
    const int lane = threadIdx.x & 31, chunks = positions * (c.dh / 8);
    const uint4 *f = reinterpret_cast<const uint4 *>(c.pool) + c.row(l, src, 0, head, 0) / 8;  // (a page's heads of V follow those of K)
    uint4 *t = reinterpret_cast<uint4 *>(c.pool) + c.row(l, dst, 0, head, 0) / 8;
    for (int c0 = lane; c0 < chunks; c0 += 8 * 32) {
        uint4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + 32 * e < chunks) v[e] = ldg_stream16(f + c0 + 32 * e);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + 32 * e < chunks) t[c0 + 32 * e] = v[e];
    }
}

// Bound by its dependent passes - tables and refs copied, entries given back, free ids counted, then handed out - with a barrier of the cluster
// behind each: 256 sequences of 2048 pages on 65536 ids 17 us, one sequence 5.3 (one CTA).
__global__ void __launch_bounds__(kPgThreads) pages_advance_kernel(const PagesArgs a) {
    __shared__ PagesShared s;
    cg::cluster_group cluster = cg::this_cluster();
    const int S = a.c.n_seqs, P = a.c.max_pages, N = a.c.n_pages, lg = a.c.ps_log2, up = (1 << lg) - 1, lane = threadIdx.x & 31;
    const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), thread = rank * kPgThreads + threadIdx.x, threads = ctas * kPgThreads;
    const bool wide = (int64_t)S * P > INT32_MAX;
    if (threadIdx.x == 0) s.bad = s.full = s.odd = 0, s.wanted = 0;
    if (a.table_out != a.c.table) copy_ints(a.table_out, a.c.table, (size_t)S * P, thread, threads);
    if (a.refs_out != a.refs) copy_ints(a.refs_out, a.refs, N, thread, threads);
    __syncthreads();
    // every CTA: how many pages the sequences want
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int len = a.c.lens[i], n = a.n_new[i], cap = P << lg;
        int want = 0;
        if (len < 0 || len > cap || n < 0) s.bad = 1;
        else if (n > cap - len) s.full = 1;
        else want = ((len + n + up) >> lg) - ((len + up) >> lg);
        s.prefix[i] = want;
        if (wide) atomicAdd(&s.wanted, (unsigned long long)want);
    }
    __syncthreads();
    if (wide && threadIdx.x == 0 && s.wanted > N) s.full = 1;  // (else the sums below fit 32 bits)
    const int want = scan_shared(s.prefix, S, s.part);
    cluster.sync();  // (the copies)
    // pages that no query needs any longer: a warp per sequence, from the window's first page backwards to the first that is gone
    if (a.window > 0)
        for (int i = thread >> 5; i < S; i += threads / 32) {
            const int64_t past = (int64_t)a.c.lens[i] - a.window + 1;
            const int lo = (int)(((int64_t)a.sinks + up) >> lg);
            int hi = past <= 0 ? 0 : (int)min(past >> lg, (int64_t)P);
            int32_t *row = a.table_out + (size_t)i * P;
            while (hi > lo) {
                const int j = hi - 1 - lane, page = j >= lo ? __ldcg(row + j) : -1;
                const unsigned gone = __ballot_sync(0xffffffffu, page < 0);
                if (page >= 0 && (gone & ((1u << lane) - 1u)) == 0) {
                    row[j] = -1;
                    if (page < N) atomicSub(a.refs_out + page, 1);
                    else atomicExch(cluster.map_shared_rank(&s.odd, 0), 1);
                }
                if (gone) break;
                hi -= 32;
            }
        }
    cluster.sync();
    int code = s.bad || *cluster.map_shared_rank(&s.odd, 0) ? RIVER_E_BADARG : s.full ? RIVER_E_NOPAGE : RIVER_OK;
    if (code == RIVER_OK && want > 0 &&
        !lowest_free(a.refs_out, N, want, s, cluster, [&](int k, int p) {
            const int i = owner_of(s.prefix, S, k);
            a.table_out[(size_t)i * P + ((a.c.lens[i] + up) >> lg) + k - s.prefix[i]] = p;
            a.refs_out[p] = 1;
        }))
        code = RIVER_E_NOPAGE;
    cluster.sync();  // (lens_out may be lens; `odd` has been read)
    for (int i = thread; i < S; i += threads) {
        const int len = a.c.lens[i];
        a.lens_out[i] = code == RIVER_OK ? len + a.n_new[i] : len;
    }
    if (thread == 0) *a.status = code;
}

// The same kind of passes, what a sequence needs of the others in every CTA's shared memory: 256 sequences of 26 pages 12 us, four 8.
__global__ void __launch_bounds__(kPgThreads) pages_reorder_kernel(const PagesArgs a) {
    extern __shared__ int pg_raw[];
    __shared__ PagesScan s;
    cg::cluster_group cluster = cg::this_cluster();
    const int S = a.c.n_seqs, P = a.c.max_pages, N = a.c.n_pages, lg = a.c.ps_log2, up = (1 << lg) - 1;
    const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), thread = rank * kPgThreads + threadIdx.x, threads = ctas * kPgThreads;
    // every CTA for itself: parents, lengths, the lowest child of a parent, the page that a sequence copies (-1: none), copies before its own
    int *const parent = pg_raw, *const len = parent + S, *const elder = len + S, *const src = elder + S, *const start = src + S;
    pdl_launch();
    if (threadIdx.x == 0) s.bad = s.odd = 0;
    copy_ints(a.refs_out, a.refs, N, thread, threads);
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        parent[i] = a.parents[i];
        len[i] = a.c.lens[i];
        elder[i] = S;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int p = parent[i], n = len[i];
        if (p < -1 || p >= S || n < 0 || n > (P << lg)) s.bad = 1;
        else if (p >= 0) atomicMin(&elder[p], i);
    }
    __syncthreads();
    int code = s.bad ? RIVER_E_BADARG : RIVER_OK;  // (the same in every CTA)
    int want = 0;
    if (code == RIVER_OK)
        for (int i0 = 0; i0 < S; i0 += kPgThreads) {
            const int i = i0 + threadIdx.x, p = i < S ? parent[i] : -1;
            int page = -1, total;
            if (p >= 0 && (len[p] & up) && elder[p] != i) page = a.c.table[(size_t)p * P + (len[p] >> lg)];  // the last page, another child keeps it
            const int before = cta_scan(page >= 0, s.part, total);
            if (i < S) {
                src[i] = page;
                start[i] = want + before;
            }
            want += total;
        }
    cluster.sync();  // (refs are copied)
    if (code == RIVER_OK) {
        // a warp per sequence
        for (int i = thread >> 5; i < S; i += threads / 32) {
            const int p = parent[i], old_n = (len[i] + up) >> lg, n = ((p >= 0 ? len[p] : 0) + up) >> lg, at = src[i] >= 0 ? len[p] >> lg : -1;
            const int32_t *old_row = a.c.table + (size_t)i * P, *row = a.c.table + (size_t)max(p, 0) * P;
            int32_t *to = a.table_out + (size_t)i * P;
            for (int j = threadIdx.x & 31; j < P; j += 32) {
                const int old = j < old_n ? old_row[j] : -1;
                int page = j < n ? row[j] : -1;
                if (page >= N || old >= N) {
                    atomicExch(cluster.map_shared_rank(&s.odd, 0), 1);
                    continue;
                }
                if (j == at) page = -1;  // (until the copy has an id)
                to[j] = page;
                if (page == old) continue;  // (a sequence that goes on as it was)
                if (page >= 0) atomicAdd(a.refs_out + page, 1);
                if (old >= 0) atomicSub(a.refs_out + old, 1);
            }
        }
        cluster.sync();
        code = *cluster.map_shared_rank(&s.odd, 0) ? RIVER_E_BADARG : RIVER_OK;
        if (code == RIVER_OK && want > 0 &&
            !lowest_free(a.refs_out, N, want, s, cluster, [&](int k, int id) {
                const int i = owner_of(start, S, k), n = len[parent[i]];
                int32_t *l = a.list + 1 + 3 * k;
                l[0] = src[i];
                l[1] = id;
                l[2] = n & up;
                a.table_out[(size_t)i * P + (n >> lg)] = id;
                a.refs_out[id] = 1;
            }))
            code = RIVER_E_NOPAGE;
        if (thread == 0) a.list[0] = code == RIVER_OK ? want : 0;
    } else if (thread == 0) {
        a.list[0] = 0;
    }
    if (code != RIVER_OK) {  // the state as it was
        cluster.sync();
        copy_ints(a.table_out, a.c.table, (size_t)S * P, thread, threads);
        copy_ints(a.refs_out, a.refs, N, thread, threads);
    }
    for (int i = thread; i < S; i += threads) {
        const int p = parent[i];
        a.lens_out[i] = code != RIVER_OK ? len[i] : p >= 0 ? len[p] : 0;
    }
    if (thread == 0) *a.status = code;
    cluster.sync();  // (nobody leaves while its shared memory may be read; the list is written)
    if (a.copy_here && code == RIVER_OK) {
        const int heads = 2 * a.c.Hkv, L = a.c.n_layers;
        for (int w = thread >> 5; w < want * L * heads; w += threads / 32) {
            const int *e = a.list + 1 + 3 * (w / heads / L);
            copy_head(a.c, w / heads % L, w % heads, __ldcg(e), __ldcg(e + 1), __ldcg(e + 2));
        }
    }
}

// Two passes over refs and one over the moves: 2048 ids 8.4 us.
__global__ void __launch_bounds__(kPgThreads) pages_compact_kernel(const PagesArgs a) {
    __shared__ PagesScan s;
    cg::cluster_group cluster = cg::this_cluster();
    const int N = a.c.n_pages, rank = cluster.block_rank(), ctas = cluster.num_blocks(), thread = rank * kPgThreads + threadIdx.x, threads = ctas * kPgThreads;
    const Run run(N, rank, ctas);
    int32_t *to = a.list + 1, *from = to + N / 2;
    pdl_launch();
    int mine = 0, used;
    run.each(a.refs, [&](int, int r) { mine += r > 0; });
    int u = cluster_scan(mine, s, cluster, used);
    // Page q has u used ones before it.  Below `used` a page that is free is hole number q - u; from there on the used ones are the movers,
    // numbered from behind for now: how many they are is known when page used - 1 has been seen.
    run.each(a.refs, [&](int q, int r) {
        const bool in_use = r > 0;
        if (q < used && !in_use) to[q - u] = q;
        if (q >= used && in_use) from[N / 2 - (used - u)] = q;
        a.remap[q] = in_use ? q : -1;
        if (a.refs_out != a.refs) a.refs_out[q] = r;
        u += in_use;
        if (q == used - 1) *cluster.map_shared_rank(&s.count[1], 0) = used - u;
    });
    if (used == 0 && thread == 0) s.count[1] = 0;
    cluster.sync();
    const int moves = *cluster.map_shared_rank(&s.count[1], 0);
    const int32_t *last = from + N / 2 - moves;  // the movers, ascending
    for (int k = thread; k < moves; k += threads) {
        const int f = __ldcg(last + k), t = __ldcg(to + k);
        a.remap[f] = t;
        a.refs_out[t] = __ldcg(a.refs + f);
    }
    cluster.sync();
    // the list's second part begins at its first place (a copy to itself where nothing is left over)
    for (int k0 = 0; k0 < moves; k0 += threads) {
        const int k = k0 + thread, f = k < moves ? __ldcg(last + k) : 0;
        cluster.sync();
        if (k < moves) {
            from[k] = f;
            a.refs_out[f] = 0;
        }
        cluster.sync();
    }
    if (thread == 0) { *a.n_used = used; a.list[0] = moves; }
}

// The values of the pages on the list, a warp per (page, block, head): triples: (from, to, positions) entries; else whole
// pages, to[] and from[] apart, and the table's entries follow `remap`.
// Bound by HBM: 2 GB of whole pages 309 us with the deciding kernel, 6.3 TB/s (97 % of a plain copy); 233 MB of pages in parts 42 us.
constexpr int kCopyCtas = 64;  // of the grid, per SM (8 are resident; grids of 8, 32 and 64 take 330, 312, 309 us for 2 GB)
__global__ void __launch_bounds__(256) pages_copy_kernel(const PagesArgs a, int triples) {
    pdl_wait();
    const int n = a.list[0], heads = 2 * a.c.Hkv, warps = gridDim.x * 8, L = a.c.n_layers;
    for (int64_t w = blockIdx.x * 8 + (threadIdx.x >> 5); w < (int64_t)n * L * heads; w += warps) {
        const int head = (int)(w % heads), l = (int)(w / heads % L), k = (int)(w / heads / L);
        const int src = triples ? a.list[1 + 3 * k] : a.list[1 + a.c.n_pages / 2 + k], dst = triples ? a.list[2 + 3 * k] : a.list[1 + k];
        copy_head(a.c, l, head, src, dst, triples ? a.list[3 + 3 * k] : 1 << a.c.ps_log2);
    }
    if (triples) return;
    const size_t entries = (size_t)a.c.n_seqs * a.c.max_pages;
    for (size_t e = blockIdx.x * 256 + threadIdx.x; e < entries; e += (size_t)gridDim.x * 256) {
        const int page = a.c.table[e];
        a.table_out[e] = page >= 0 && page < a.c.n_pages ? a.remap[page] : -1;
    }
}

// work: table entries and page ids.  A few thousand are one CTA's; from 2^18 on twice the portable cluster pays (256 sequences of 2048
// pages, 65536 ids: 24 -> 17 us).
template <class K>
int launch_deciding(K kernel, const PagesArgs &a, size_t work, size_t smem, cudaStream_t st) {
    const unsigned ctas = work <= 4 * kPgThreads ? 1 : work < (1u << 18) ? kPgCtas : 2 * kPgCtas;
    if (ctas > 8 && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return RIVER_E_DEVICE;
    // the limit belongs to the kernel, not to the call: whoever sets it sets the same one, or a launch of another thread could fail by it
    constexpr int most = kPgSeqInts * sizeof(int) * kPgSeqs;
    if (smem > (32u << 10) && cuda_rc(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most))) return RIVER_E_DEVICE;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {ctas, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPgThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = ctas > 1 ? 1 : 0;
    return cuda_rc(cudaLaunchKernelEx(&cfg, kernel, a));
}
// `most`: heads' worth of copies that there may be
int launch_copy(const PagesArgs &a, int triples, int64_t most, cudaStream_t st) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;  // (its CTAs stand ready when the list is there)
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<int64_t>(148 * kCopyCtas, std::max<int64_t>(1, (most + 7) / 8)));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cuda_rc(cudaLaunchKernelEx(&cfg, pages_copy_kernel, a, triples));
}

}  // namespace
}  // namespace river

using namespace river;

extern "C" int river_pages_advance(const river_paged *c, const int32_t *refs, const int32_t *n_new, int window, int sinks, int32_t *table_out,
                                   int32_t *lens_out, int32_t *refs_out, int32_t *status, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, false, true, &a.c)) return rc;
    if (!refs || !n_new || !table_out || !lens_out || !refs_out || !status || window < 0 || sinks < 0) return RIVER_E_BADARG;
    if (!words(refs, n_new, table_out, lens_out, refs_out, status)) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs) return RIVER_E_SHAPE;
    a.refs = refs;
    a.n_new = n_new;
    a.window = window;
    a.sinks = sinks;
    a.table_out = table_out;
    a.lens_out = lens_out;
    a.refs_out = refs_out;
    a.status = status;
    return launch_deciding(pages_advance_kernel, a, (size_t)c->n_seqs * c->max_pages + c->n_pages, 0, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int river_pages_reorder(const river_paged *c, const int32_t *refs, const int32_t *parents, int32_t *table_out, int32_t *lens_out,
                                   int32_t *refs_out, int32_t *copies, int32_t *status, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, true, true, &a.c)) return rc;
    if (!refs || !parents || !table_out || !lens_out || !refs_out || !copies || !status) return RIVER_E_BADARG;
    if (!words(refs, parents, table_out, lens_out, refs_out, copies, status)) return RIVER_E_BADARG;
    if (table_out == c->table || lens_out == c->lens || refs_out == refs) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs) return RIVER_E_SHAPE;
    a.refs = refs;
    a.parents = parents;
    a.table_out = table_out;
    a.lens_out = lens_out;
    a.refs_out = refs_out;
    a.list = copies;
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    // A few sequences' last pages (up to 4 MB) are copied by the deciding cluster itself, which saves the host a launch: four beams of the 1B class 14.2 us
    // in two launches, 12.3 in one.  The GPU alone takes longer that way (in a graph, us in one / two: 0.25 MB 10.7 / 7.6, 2 MB 13.5 / 7.6, 4 MB 19.1 /
    // 8.4, 8 MB 30.5 / 9.7), and at 4 MB the host's launch costs less than that (20.6 / 16 in a loop).
    const int64_t most = (int64_t)std::min(c->n_seqs, c->n_pages) * c->n_layers * 2 * c->Hkv;
    a.copy_here = most * c->page_size * c->dh * 2 <= (4 << 20);
    const size_t work = std::max((size_t)c->n_seqs * c->max_pages + c->n_pages, a.copy_here && most > 32 ? (size_t)4 * kPgThreads + 1 : (size_t)0);
    if (const int rc = launch_deciding(pages_reorder_kernel, a, work, kPgSeqInts * sizeof(int) * (size_t)c->n_seqs, st)) return rc;
    return a.copy_here ? RIVER_OK : launch_copy(a, 1, most, st);
}

extern "C" int river_pages_compact(const river_paged *c, const int32_t *refs, int32_t *table_out, int32_t *refs_out, int32_t *remap,
                                   int32_t *n_used, int32_t *moves, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, true, false, &a.c)) return rc;
    if (!refs || !table_out || !refs_out || !remap || !n_used || !moves) return RIVER_E_BADARG;
    if (!words(refs, table_out, refs_out, remap, n_used, moves)) return RIVER_E_BADARG;
    a.refs = refs;
    a.table_out = table_out;
    a.refs_out = refs_out;
    a.remap = remap;
    a.n_used = n_used;
    a.list = moves;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (const int rc = launch_deciding(pages_compact_kernel, a, c->n_pages, 0, st)) return rc;
    return launch_copy(a, 0, (int64_t)c->n_pages / 2 * c->n_layers * 2 * c->Hkv + (int64_t)c->n_seqs * c->max_pages / 32, st);
}

// river_pages_advance, river_pages_reorder, river_pages_compact: the pages of a paged cache, kept on the device.
//
// Which page goes where is decided by one CTA: a few prefix sums over sequences and page ids.  Free pages are those with refs 0 after
// what the call gives back; the k-th page that is wanted, in order of (sequence, position), receives the k-th free id.  The values
// then move in a kernel of their own that reads the list of copies.
#include "paged_common.cuh"

namespace river {
namespace {

constexpr int kPgThreads = 1024;
constexpr int kPgSeqs = 8192;  // sequences whose prefix sums are held in shared memory

struct PagesArgs {
    Paged c;
    const int32_t *refs, *n_new, *parents;
    int window, sinks;
    int32_t *table_out, *lens_out, *refs_out, *list, *status;  // list: of copies or moves
    int32_t *remap, *n_used;
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

// give(k, id) for the `want` lowest ids with refs 0, ascending; returns how many there were (at most want).
template <class F>
__device__ int lowest_free(const volatile int32_t *refs, int n_pages, int want, int *part, F give) {
    int got = 0;
    for (int p0 = 0; p0 < n_pages && got < want; p0 += kPgThreads) {
        const int p = p0 + threadIdx.x;
        const bool free_ = p < n_pages && refs[p] == 0;
        int total;
        const int k = got + cta_scan(free_, part, total);
        if (free_ && k < want) give(k, p);
        got += total;
    }
    __syncthreads();
    return min(got, want);
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

__global__ void __launch_bounds__(kPgThreads) pages_advance_kernel(const PagesArgs a) {
    __shared__ int part[33], s_bad, s_full, prefix[kPgSeqs];
    const int S = a.c.n_seqs, P = a.c.max_pages, N = a.c.n_pages, lg = a.c.ps_log2, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) s_bad = s_full = 0;
    if (a.table_out != a.c.table)
        for (size_t i = threadIdx.x; i < (size_t)S * P; i += kPgThreads) a.table_out[i] = a.c.table[i];
    if (a.refs_out != a.refs)
        for (int p = threadIdx.x; p < N; p += kPgThreads) a.refs_out[p] = a.refs[p];
    __syncthreads();
    // pages that no query needs any longer: a warp per sequence, from the window's first page backwards to the first that is gone
    if (a.window > 0)
        for (int s = threadIdx.x >> 5; s < S; s += kPgThreads / 32) {
            const int64_t past = (int64_t)a.c.lens[s] - a.window + 1;
            const int lo = (a.sinks + (1 << lg) - 1) >> lg;
            int hi = past <= 0 ? 0 : (int)min(past >> lg, (int64_t)P);
            int32_t *row = a.table_out + (size_t)s * P;
            while (hi > lo) {
                const int j = hi - 1 - lane, page = j >= lo ? row[j] : -1;
                const unsigned gone = __ballot_sync(0xffffffffu, page < 0);
                if (page >= 0 && (gone & ((1u << lane) - 1u)) == 0) {
                    row[j] = -1;
                    if (page < N) atomicSub(a.refs_out + page, 1);
                    else s_bad = 1;
                }
                if (gone) break;
                hi -= 32;
            }
        }
    for (int s = threadIdx.x; s < S; s += kPgThreads) {
        const int len = a.c.lens[s], n = a.n_new[s], cap = P << lg;
        int want = 0;
        if (len < 0 || len > cap || n < 0) s_bad = 1;
        else if (n > cap - len) s_full = 1;
        else want = ((len + n + (1 << lg) - 1) >> lg) - ((len + (1 << lg) - 1) >> lg);
        prefix[s] = want;
    }
    __syncthreads();
    const int bad = s_bad, full = s_full, want = scan_shared(prefix, S, part);
    int code = bad ? RIVER_E_BADARG : full ? RIVER_E_NOPAGE : RIVER_OK;
    if (code == RIVER_OK) {
        auto entry = [&](int k) {
            const int s = owner_of(prefix, S, k);
            return a.table_out + (size_t)s * P + ((a.c.lens[s] + (1 << lg) - 1) >> lg) + k - prefix[s];
        };
        const int got = lowest_free(a.refs_out, N, want, part, [&](int k, int p) { *entry(k) = p; });
        for (int k = threadIdx.x; k < got; k += kPgThreads) {  // (behind the scan, which reads refs)
            if (got == want) a.refs_out[*entry(k)] = 1;
            else *entry(k) = -1;
        }
        if (got < want) code = RIVER_E_NOPAGE;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < S; s += kPgThreads) {
        const int len = a.c.lens[s];
        a.lens_out[s] = code == RIVER_OK ? len + a.n_new[s] : len;
    }
    if (threadIdx.x == 0) *a.status = code;
}

__global__ void __launch_bounds__(kPgThreads) pages_reorder_kernel(const PagesArgs a) {
    __shared__ int part[33], s_bad, elder[kPgSeqs];  // elder: the lowest child of a parent, then prefix sums of the copies
    const int S = a.c.n_seqs, P = a.c.max_pages, N = a.c.n_pages, lg = a.c.ps_log2, ps = 1 << lg;
    if (threadIdx.x == 0) s_bad = 0;
    for (int s = threadIdx.x; s < S; s += kPgThreads) elder[s] = S;
    for (int p = threadIdx.x; p < N; p += kPgThreads) a.refs_out[p] = a.refs[p];
    __syncthreads();
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int p = a.parents[i], len = a.c.lens[i];
        if (p < -1 || p >= S || len < 0 || len > (P << lg)) s_bad = 1;
        else if (p >= 0) atomicMin(&elder[p], i);
    }
    __syncthreads();
    int code = s_bad ? RIVER_E_BADARG : RIVER_OK;
    if (code == RIVER_OK) {
        // a sequence that copies its last page, filled in part
        auto copies = [&](int i, int p) { return p >= 0 && (a.c.lens[p] & (ps - 1)) && elder[p] != i; };
        for (size_t e = threadIdx.x; e < (size_t)S * P; e += kPgThreads) {
            const int i = (int)(e / P), j = (int)(e % P), p = a.parents[i];
            const int old = j < (a.c.lens[i] + ps - 1) >> lg ? a.c.table[e] : -1;
            int page = -1;
            if (p >= 0 && j < (a.c.lens[p] + ps - 1) >> lg) page = a.c.table[(size_t)p * P + j];
            if (page >= N || old >= N) { s_bad = 1; continue; }
            const bool own_copy = j == (p >= 0 ? a.c.lens[p] >> lg : -1) && copies(i, p);
            if (own_copy) page = page < 0 ? -1 : -2 - page;  // (the page to copy from, until its copy has an id)
            a.table_out[e] = page;
            if (page == old) continue;  // (a sequence that goes on as it was)
            if (page >= 0) atomicAdd(a.refs_out + page, 1);
            if (old >= 0) atomicSub(a.refs_out + old, 1);
        }
        __syncthreads();
        code = s_bad ? RIVER_E_BADARG : RIVER_OK;
        __syncthreads();
        for (int i = threadIdx.x; i < S; i += kPgThreads) {
            const int p = a.parents[i];
            elder[i] = p >= 0 && (a.c.lens[p] & (ps - 1)) && a.table_out[(size_t)i * P + (a.c.lens[p] >> lg)] < -1;
        }
        __syncthreads();
    }
    if (code == RIVER_OK) {
        const int want = scan_shared(elder, S, part);
        const int got = lowest_free(a.refs_out, N, want, part, [&](int k, int id) {
            const int i = owner_of(elder, S, k), p = a.parents[i];
            int32_t *e = a.table_out + (size_t)i * P + (a.c.lens[p] >> lg), *l = a.list + 1 + 3 * k;
            l[0] = -2 - *e;
            l[1] = id;
            l[2] = a.c.lens[p] & (ps - 1);
            *e = id;
        });
        for (int k = threadIdx.x; k < got; k += kPgThreads) a.refs_out[a.list[2 + 3 * k]] = 1;
        if (threadIdx.x == 0) a.list[0] = got == want ? got : 0;
        if (got < want) code = RIVER_E_NOPAGE;
    }
    if (code != RIVER_OK) {
        __syncthreads();
        for (size_t e = threadIdx.x; e < (size_t)S * P; e += kPgThreads) a.table_out[e] = a.c.table[e];
        for (int p = threadIdx.x; p < N; p += kPgThreads) a.refs_out[p] = a.refs[p];
        if (threadIdx.x == 0) a.list[0] = 0;
    }
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int p = a.parents[i];
        a.lens_out[i] = code != RIVER_OK ? a.c.lens[i] : p >= 0 ? a.c.lens[p] : 0;
    }
    if (threadIdx.x == 0) *a.status = code;
}

__global__ void __launch_bounds__(kPgThreads) pages_compact_kernel(const PagesArgs a) {
    __shared__ int part[33];
    const int N = a.c.n_pages;
    int32_t *to = a.list + 1, *from = to + N / 2;
    int used = 0;
    for (int p0 = 0; p0 < N; p0 += kPgThreads) {
        const int p = p0 + threadIdx.x;
        int total;
        cta_scan(p < N && a.refs[p] > 0, part, total);
        used += total;
    }
    int holes = 0, movers = 0;
    for (int p0 = 0; p0 < N; p0 += kPgThreads) {
        const int p = p0 + threadIdx.x, r = p < N ? a.refs[p] : 0;
        const bool hole = p < used && r <= 0, mover = p >= used && r > 0;
        int nh, nm;
        const int h = cta_scan(hole, part, nh), m = cta_scan(mover, part, nm);
        if (hole) to[holes + h] = p;
        if (mover) from[movers + m] = p;
        if (p < N) {
            a.remap[p] = r > 0 ? p : -1;
            if (a.refs_out != a.refs) a.refs_out[p] = r;
        }
        holes += nh;
        movers += nm;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < movers; k += kPgThreads) {
        a.remap[from[k]] = to[k];
        a.refs_out[to[k]] = a.refs_out[from[k]];
        a.refs_out[from[k]] = 0;
    }
    __syncthreads();
    for (size_t e = threadIdx.x; e < (size_t)a.c.n_seqs * a.c.max_pages; e += kPgThreads) {
        const int page = a.c.table[e];
        a.table_out[e] = page >= 0 && page < N ? a.remap[page] : -1;
    }
    if (threadIdx.x == 0) { *a.n_used = used; a.list[0] = movers; }
}

// The values of the pages on the list, layer by layer.  triples: (from, to, positions) entries, of which the first `positions` of every
// head move; else whole pages, to[] and from[] apart.
__global__ void __launch_bounds__(256) pages_copy_kernel(const Paged c, const int32_t *list, int triples) {
    const int n = list[0], heads = 2 * c.Hkv;
    for (int u = blockIdx.x; u < n * c.n_layers; u += gridDim.x) {
        const int k = u / c.n_layers, l = u % c.n_layers;
        const int src = triples ? list[1 + 3 * k] : list[1 + c.n_pages / 2 + k], dst = triples ? list[2 + 3 * k] : list[1 + k];
        const int fill = triples ? list[3 + 3 * k] : 1 << c.ps_log2, chunks = fill * (c.dh / 8);  // 16-byte chunks of a head
        const uint4 *s = reinterpret_cast<const uint4 *>(c.pool) + c.row(l, src, 0, 0, 0) / 8;
        uint4 *d = reinterpret_cast<uint4 *>(c.pool) + c.row(l, dst, 0, 0, 0) / 8;
        for (int i = threadIdx.x; i < heads * chunks; i += blockDim.x) {
            const int at = i / chunks * ((c.dh / 8) << c.ps_log2) + i % chunks;
            d[at] = s[at];
        }
    }
}

}  // namespace
}  // namespace river

using namespace river;

extern "C" int river_pages_advance(const river_paged *c, const int32_t *refs, const int32_t *n_new, int window, int sinks, int32_t *table_out,
                                   int32_t *lens_out, int32_t *refs_out, int32_t *status, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, false, true, &a.c)) return rc;
    if (!refs || !n_new || !table_out || !lens_out || !refs_out || !status || window < 0 || sinks < 0) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs) return RIVER_E_SHAPE;
    a.refs = refs;
    a.n_new = n_new;
    a.window = window;
    a.sinks = sinks;
    a.table_out = table_out;
    a.lens_out = lens_out;
    a.refs_out = refs_out;
    a.status = status;
    pages_advance_kernel<<<1, kPgThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    return launch_rc();
}

extern "C" int river_pages_reorder(const river_paged *c, const int32_t *refs, const int32_t *parents, int32_t *table_out, int32_t *lens_out,
                                   int32_t *refs_out, int32_t *copies, int32_t *status, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, true, true, &a.c)) return rc;
    if (!refs || !parents || !table_out || !lens_out || !refs_out || !copies || !status) return RIVER_E_BADARG;
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
    pages_reorder_kernel<<<1, kPgThreads, 0, st>>>(a);
    pages_copy_kernel<<<148 * 8, 256, 0, st>>>(a.c, copies, 1);
    return launch_rc();
}

extern "C" int river_pages_compact(const river_paged *c, const int32_t *refs, int32_t *table_out, int32_t *refs_out, int32_t *remap,
                                   int32_t *n_used, int32_t *moves, void *cuda_stream) {
    PagesArgs a = {};
    if (const int rc = paged_check(c, true, false, &a.c)) return rc;
    if (!refs || !table_out || !refs_out || !remap || !n_used || !moves) return RIVER_E_BADARG;
    a.refs = refs;
    a.table_out = table_out;
    a.refs_out = refs_out;
    a.remap = remap;
    a.n_used = n_used;
    a.list = moves;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    pages_compact_kernel<<<1, kPgThreads, 0, st>>>(a);
    pages_copy_kernel<<<148 * 8, 256, 0, st>>>(a.c, moves, 0);
    return launch_rc();
}

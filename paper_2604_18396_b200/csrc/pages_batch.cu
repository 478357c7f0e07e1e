// river_pages_admit, river_pages_slots, river_prefix_groups: the page tables of a batch of requests from their lengths, the places of its new
// tokens, and which of its sequences share their first pages.
#include "pages_scan.cuh"

namespace river {
namespace {

// Adds n of every thread to *to (shared memory), an addition per warp.  All threads of the warp.
__device__ __forceinline__ void add_wide(unsigned long long *to, long long n) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if ((threadIdx.x & 31) == 0 && n) atomicAdd(to, (unsigned long long)n);
}

struct AdmitArgs {
    Paged c;
    const int32_t *refs, *like, *begin, *total;
    int32_t *table_out, *lens_out, *refs_out, *n_new, *status;
    int rest;  // the entries behind the requests' pages are another kernel's
};

// Table entries behind a request's pages, by all SMs, beside the deciding cluster.
__global__ void __launch_bounds__(256) pages_admit_rest_kernel(const AdmitArgs a) {
    pdl_launch();
    const int P = a.c.max_pages, up = (1 << a.c.ps_log2) - 1;
    for (int i = blockIdx.x; i < a.c.n_seqs; i += gridDim.x) {
        const int64_t total = max(0, a.total[i]);
        for (int64_t j = ((total + up) >> a.c.ps_log2) + threadIdx.x; j < P; j += 256) a.table_out[(size_t)i * P + j] = -1;
    }
}

// Passes like those of pages_reorder_kernel (pages.cu): refs copied, rows written with their entries counted, free ids counted, then handed out.
// Bound by them, and by what 16 SMs read and write in them: 512 sequences of 2048 pages on 262144 ids 44 us with a row's entries 32 at a time and the
// lowest ids given by the cluster's first CTA, 30 with 512 entries and every CTA giving, 20 with the empty entries left to the other SMs.
constexpr int kAdUnder = 16;  // times 32 entries of a row under way
__global__ void __launch_bounds__(kPgThreads) pages_admit_kernel(const AdmitArgs a) {
    extern __shared__ int pg_raw[];
    __shared__ PagesScan s;
    cg::cluster_group cluster = cg::this_cluster();
    const int S = a.c.n_seqs, P = a.c.max_pages, N = a.c.n_pages, lg = a.c.ps_log2, up = (1 << lg) - 1, cap = P << lg;
    const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), thread = rank * kPgThreads + threadIdx.x, threads = ctas * kPgThreads;
    // every CTA for itself: whom a request begins like, lengths held and wanted, positions that it begins with, pages wanted before its own
    int *const like = pg_raw, *const len = like + S, *const total = len + S, *const keep = total + S, *const start = keep + S;
    if (threadIdx.x == 0) s.bad = s.full = s.odd = 0, s.wanted = 0;
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        like[i] = a.like[i];
        len[i] = a.c.lens[i];
        total[i] = a.total[i];
        keep[i] = a.begin[i];
    }
    copy_ints(a.refs_out, a.refs, N, thread, threads);
    __syncthreads();
    long long mine = 0;
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int p = like[i], b = keep[i], n = total[i];
        int k = 0, want = 0;
        if (p < -1 || p >= S || b < 0 || n < 0 || len[i] < 0 || len[i] > cap) s.bad = 1;
        else if (n > cap) s.full = 1;
        else {
            k = p < 0 ? 0 : max(0, min(min(b, len[p]), n));
            if (p != i || k != len[i]) k &= ~up;  // (a page that is filled in part is nobody else's)
            want = ((n + up) >> lg) - ((k + up) >> lg);
        }
        keep[i] = k;
        start[i] = want;
        mine += want;
    }
    add_wide(&s.wanted, mine);
    __syncthreads();
    if (threadIdx.x == 0 && s.wanted > N) s.full = 1;  // (else the sums below fit 32 bits)
    __syncthreads();
    int code = s.bad ? RIVER_E_BADARG : s.full ? RIVER_E_NOPAGE : RIVER_OK;  // (the same in every CTA)
    int want = 0;
    if (code == RIVER_OK) want = scan_shared(start, S, s.part);
    cluster.sync();  // (refs are copied)
    if (code == RIVER_OK) {
        // a warp per sequence
        for (int i = thread >> 5; i < S; i += threads / 32) {
            const int old_n = (len[i] + up) >> lg, n = (keep[i] + up) >> lg, end = a.rest ? max(old_n, n) : P, mine_to = (total[i] + up) >> lg;
            const int32_t *old_row = a.c.table + (size_t)i * P, *row = a.c.table + (size_t)max(like[i], 0) * P;
            int32_t *to = a.table_out + (size_t)i * P;
            for (int j0 = threadIdx.x & 31; j0 < end; j0 += 32 * kAdUnder) {
                int old[kAdUnder], page[kAdUnder];
#pragma unroll
                for (int e = 0; e < kAdUnder; ++e) {
                    const int j = j0 + 32 * e;
                    old[e] = j < old_n ? old_row[j] : -1;
                    page[e] = j < n ? max(row[j], -1) : -1;
                }
#pragma unroll
                for (int e = 0; e < kAdUnder; ++e) {
                    const int j = j0 + 32 * e;
                    if (j >= end) continue;
                    if (page[e] >= N || old[e] >= N) {
                        atomicExch(cluster.map_shared_rank(&s.odd, 0), 1);
                        continue;
                    }
                    if (!a.rest || j < mine_to) to[j] = page[e];
                    if (page[e] == old[e]) continue;  // (a sequence that goes on)
                    if (page[e] >= 0) atomicAdd(a.refs_out + page[e], 1);
                    if (old[e] >= 0) atomicSub(a.refs_out + old[e], 1);
                }
            }
        }
        cluster.sync();
        code = *cluster.map_shared_rank(&s.odd, 0) ? RIVER_E_BADARG : RIVER_OK;
        if (code == RIVER_OK && want > 0 &&
            !lowest_free(a.refs_out, N, want, s, cluster, [&](int k, int id) {
                const int i = owner_of(start, S, k);
                a.table_out[(size_t)i * P + ((keep[i] + up) >> lg) + k - start[i]] = id;
                a.refs_out[id] = 1;
            }))
            code = RIVER_E_NOPAGE;
    }
    if (a.rest) pdl_wait();  // (the other entries are written; and this kernel ends behind that one)
    if (code != RIVER_OK) {  // the state as it was
        cluster.sync();
        copy_ints(a.table_out, a.c.table, (size_t)S * P, thread, threads);
        copy_ints(a.refs_out, a.refs, N, thread, threads);
    }
    for (int i = thread; i < S; i += threads) {
        a.lens_out[i] = code == RIVER_OK ? total[i] : len[i];
        a.n_new[i] = code == RIVER_OK ? total[i] - keep[i] : 0;
    }
    if (thread == 0) *a.status = code;
    cluster.sync();  // (nobody leaves while its shared memory may be read)
}

struct SlotsArgs {
    Paged c;
    const int32_t *n_new;
    int n_tokens;
    int32_t *q_start, *positions, *seqs;
    int64_t *slots;
    int32_t *status;
};

// Every CTA sums up the batch for itself; a thread then finds its tokens' sequences among the sums.  Bound by those steps one after the other: 8 sequences with
// a token each 4.6 us, 256 with up to 512 each 6.
constexpr int kSlTokens = 2;  // of a thread
__global__ void __launch_bounds__(kPgThreads) pages_slots_kernel(const SlotsArgs a) {
    __shared__ PagesShared s;
    const int S = a.c.n_seqs, lg = a.c.ps_log2;
    if (threadIdx.x == 0) s.bad = 0, s.wanted = 0;
    __syncthreads();
    long long mine = 0;
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int n = a.n_new[i];
        if (n < 0) s.bad = 1;
        s.prefix[i] = min(max(n, 0), a.n_tokens);
        mine += max(n, 0);
    }
    add_wide(&s.wanted, mine);
    __syncthreads();
    const bool fits = s.wanted <= (unsigned long long)a.n_tokens;  // (else nothing has a place)
    const int all = fits ? scan_shared(s.prefix, S, s.part) : 0;
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i <= S; i += kPgThreads) a.q_start[i] = !fits ? 0 : i < S ? s.prefix[i] : all;
        if (threadIdx.x == 0 && (s.bad || !fits)) flag(a.status, RIVER_E_BADARG);
    }
    for (int t = blockIdx.x * kPgThreads + threadIdx.x; t < a.n_tokens; t += gridDim.x * kPgThreads) {
        int seq = -1, pos = -1;
        int64_t slot = -1;
        if (t < all) {
            seq = owner_of(s.prefix, S, t);
            const int n = a.n_new[seq], len = a.c.lens[seq];
            pos = len - n + t - s.prefix[seq];
            const int col = pos >> lg, page = pos >= 0 && len >= 0 && col < a.c.max_pages ? a.c.table[(size_t)seq * a.c.max_pages + col] : -1;
            if (page >= 0) slot = ((int64_t)page << lg) + (pos & ((1 << lg) - 1));
            else flag(a.status, RIVER_E_BADARG);
        }
        a.positions[t] = pos;
        a.seqs[t] = seq;
        a.slots[t] = slot;
    }
}

struct GroupsArgs {
    Paged c;
    const int32_t *q_start;
    int least;
    int32_t *lead, *shared;
};
constexpr int kGrSmall = 16384;  // table entries that one CTA compares by itself

// Equal first entries of the rows of sequences i - 1 and i, among those of whole pages that both held before their new tokens.  A warp.
__device__ __forceinline__ int equal_pages(const GroupsArgs &a, int i) {
    if (i == 0) return 0;
    const int P = a.c.max_pages, lane = threadIdx.x & 31;
    auto whole = [&](int s) { return (int)max((int64_t)0, min((int64_t)a.c.lens[s] - max((int64_t)0, (int64_t)a.q_start[s + 1] - a.q_start[s]), (int64_t)P << a.c.ps_log2)) >> a.c.ps_log2; };
    const int w = min(whole(i - 1), whole(i));
    const int32_t *x = a.c.table + (size_t)(i - 1) * P, *y = x + P;
    constexpr int U = 16;
    for (int j0 = 0; j0 < w; j0 += 32 * U) {
        int p[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + 32 * u + lane;
            p[u] = j < w ? x[j] : -1;
            r[u] = j < w ? y[j] : -2;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned other = __ballot_sync(0xffffffffu, p[u] != r[u] || p[u] < 0);
            if (other) return j0 + 32 * u + __ffs(other) - 1;
        }
    }
    return w;
}
// From the equal pages of neighbours, `c`, to leads and shared positions, by one CTA (prefix: n_seqs ints).
__device__ __forceinline__ void groups_of(const GroupsArgs &a, const int32_t *c, int *prefix, int *part) {
    const int S = a.c.n_seqs, lg = a.c.ps_log2, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int carry = 0;  // the first sequence of the group that is open
    for (int i0 = 0; i0 < S; i0 += kPgThreads) {
        const int i = i0 + threadIdx.x, n = i < S ? c[i] : 0;
        const bool linked = n > 0 && ((int64_t)n << lg) >= a.least;
        int l = i < S && !linked ? i : -1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, l, o);
            if (lane >= o) l = max(l, x);
        }
        if (lane == 31) part[warp] = l;
        if (i < S) prefix[i] = INT32_MAX;
        __syncthreads();
        const int first = part[lane];  // of warp `lane`
        l = max(l, max(carry, __reduce_max_sync(0xffffffffu, lane < warp ? first : -1)));
        carry = max(carry, __reduce_max_sync(0xffffffffu, first));
        if (i < S) a.lead[i] = l;
        if (linked) atomicMin(&prefix[l], n);
        __syncthreads();
    }
    for (int i = threadIdx.x; i < S; i += kPgThreads) {
        const int n = prefix[a.lead[i]];
        a.shared[i] = n == INT32_MAX ? 0 : n << lg;
    }
}

// Equal pages, a warp per sequence: 1000 rows that share 60 to 1250 pages 5.6 us.  The leads, by one CTA, 5 more, of which the start runs beside it; 8 rows by one CTA 3.5.
__global__ void __launch_bounds__(256) prefix_equal_kernel(const GroupsArgs a) {
    pdl_launch();
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (i >= a.c.n_seqs) return;
    const int n = equal_pages(a, i);
    if ((threadIdx.x & 31) == 0) a.shared[i] = n;
}
// one CTA; `small`: it compares as well
__global__ void __launch_bounds__(kPgThreads) prefix_groups_kernel(const GroupsArgs a, int small) {
    __shared__ int prefix[kPgSeqs], equal[kPgThreads], part[32];
    if (small) {
        for (int i = threadIdx.x >> 5; i < a.c.n_seqs; i += kPgThreads / 32) {
            const int n = equal_pages(a, i);
            if ((threadIdx.x & 31) == 0) equal[i] = n;
        }
        __syncthreads();
        groups_of(a, equal, prefix, part);
    } else {
        pdl_wait();
        groups_of(a, a.shared, prefix, part);
    }
}

}  // namespace
}  // namespace river

using namespace river;

extern "C" int river_pages_admit(const river_paged *c, const int32_t *refs, const int32_t *like, const int32_t *begin, const int32_t *total,
                                 int32_t *table_out, int32_t *lens_out, int32_t *refs_out, int32_t *n_new, int32_t *status, void *cuda_stream) {
    AdmitArgs a = {};
    if (const int rc = paged_check(c, false, true, &a.c)) return rc;
    if (!refs || !like || !begin || !total || !table_out || !lens_out || !refs_out || !n_new || !status) return RIVER_E_BADARG;
    if (!words(refs, like, begin, total, table_out, lens_out, refs_out, n_new, status)) return RIVER_E_BADARG;
    if (table_out == c->table || lens_out == c->lens || refs_out == refs) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs) return RIVER_E_SHAPE;
    a.refs = refs;
    a.like = like;
    a.begin = begin;
    a.total = total;
    a.table_out = table_out;
    a.lens_out = lens_out;
    a.refs_out = refs_out;
    a.n_new = n_new;
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t entries = (size_t)c->n_seqs * c->max_pages;
    a.rest = entries >= (1u << 18);
    if (a.rest)
        if (const int rc = launch_plain(pages_admit_rest_kernel, dim3(std::min(c->n_seqs, 4 * 148)), dim3(256), st, a)) return rc;
    return launch_deciding(pages_admit_kernel, a, entries + c->n_pages, kPgSeqInts * sizeof(int) * (size_t)c->n_seqs, st, a.rest);
}

extern "C" int river_pages_slots(const river_paged *c, const int32_t *n_new, int n_tokens, int32_t *q_start, int32_t *positions, int32_t *seqs,
                                 int64_t *slots, int32_t *status, void *cuda_stream) {
    SlotsArgs a = {};
    if (const int rc = paged_check(c, false, true, &a.c)) return rc;
    if (!n_new || n_tokens < 0 || !q_start || (n_tokens > 0 && (!positions || !seqs || !slots))) return RIVER_E_BADARG;
    if (!words(n_new, q_start, positions, seqs, status) || !aligned_to(slots, 8)) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs || n_tokens > INT32_MAX / 2) return RIVER_E_SHAPE;
    a.n_new = n_new;
    a.n_tokens = n_tokens;
    a.q_start = q_start;
    a.positions = positions;
    a.seqs = seqs;
    a.slots = slots;
    a.status = status;
    const int ctas = std::max(1, std::min(148, (n_tokens + kSlTokens * kPgThreads - 1) / (kSlTokens * kPgThreads)));
    return launch_plain(pages_slots_kernel, dim3(ctas), dim3(kPgThreads), static_cast<cudaStream_t>(cuda_stream), a);
}

extern "C" int river_prefix_groups(const river_paged *c, const int32_t *q_start, int least, int32_t *lead, int32_t *shared, void *cuda_stream) {
    GroupsArgs a = {};
    if (const int rc = paged_check(c, false, true, &a.c)) return rc;
    if (!q_start || least < 1 || !lead || !shared || !words(q_start, lead, shared)) return RIVER_E_BADARG;
    if (c->n_seqs > kPgSeqs) return RIVER_E_SHAPE;
    a.q_start = q_start;
    a.least = least;
    a.lead = lead;
    a.shared = shared;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int small = c->n_seqs <= kPgThreads && (int64_t)c->n_seqs * c->max_pages <= kGrSmall;
    if (!small)
        if (const int rc = launch_plain(prefix_equal_kernel, dim3((c->n_seqs + 7) / 8), dim3(256), st, a)) return rc;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(kPgThreads);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = small ? 0 : 1;
    return cuda_rc(cudaLaunchKernelEx(&cfg, prefix_groups_kernel, a, small));
}

// Windowed attention of one query row by one warp, in the order of the positions (internal).
//
// A lane holds dh / 32 dims; per visible position a product, its sum over the warp, and the running maximum and sum of the softmax
// (fp32, base 2).  Every position costs a dependent chain of some hundred cycles.
#pragma once
#include "mbar_tma.cuh"
#include "paged_common.cuh"

namespace river {

struct WindowArgs {
    Paged c;
    int layer0, n_tokens, max_q, Hq, window, sinks;
    const int32_t *q_start;
    const void *q;
    int64_t q_tok, q_head;
    float scale_log2;  // softmax scale times log2 e
    void *out;
    int32_t *status;
};

// Positions that a sequence with queries holds; a length that its row of the table cannot have is told and counts as the row's, a negative one as 0.
__device__ __forceinline__ int window_len(const WindowArgs &a, int len) {
    const int cap = a.c.max_pages << a.c.ps_log2;
    if ((len < 0 || len > cap) && threadIdx.x == 0) flag(a.status, RIVER_E_BADARG);
    return max(0, min(len, cap));
}
// the first position of the window of the query at p
__device__ __forceinline__ int window_low(int p, int window) { return p >= window ? p - window + 1 : 0; }

// token: its row in q and out; seq, pos: where it stands.  The whole warp calls it.
template <class T, int DH>
__device__ void window_attn_row(const WindowArgs &a, int token, int head, int seq, int pos) {
    constexpr int E = DH / 32;
    const int lane = threadIdx.x & 31, kvh = head / (a.Hq / a.c.Hkv), pmask = (1 << a.c.ps_log2) - 1;
    const T *q = static_cast<const T *>(a.q) + token * a.q_tok + head * a.q_head + E * lane, *pool = reinterpret_cast<const T *>(a.c.pool);
    float x[E], o[E], m = -CUDART_INF_F, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) { x[e] = to_f(q[e]) * a.scale_log2; o[e] = 0.f; }
    const int low = window_low(pos, a.window), n_sink = min(a.sinks, low);
    for (int u = 0; u < n_sink + pos + 1 - low; ++u) {
        const int j = u < n_sink ? u : low + u - n_sink, col = j >> a.c.ps_log2;
        const int page = col < a.c.max_pages ? a.c.table[(size_t)seq * a.c.max_pages + col] : -1;
        if (page < 0 || page >= a.c.n_pages) {
            if (lane == 0) flag(a.status, RIVER_E_BADARG);
            continue;
        }
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
    T *out = static_cast<T *>(a.out) + ((size_t)token * a.Hq + head) * DH + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = from_f<T>(l == 0.f ? 0.f : o[e] / l);
}

}  // namespace river

// river_rope_frequencies, river_rope_append: rotary embedding of new tokens fused with their way into the paged cache.
//
// Pair i of a head turns by a = position * inv_freq[i]:  (x, y) -> scale (x cos a - y sin a, y cos a + x sin a).  The angle is the one
// place where 32 bits do not do: at position 2^17 a float product is off by 2^-8 rad, as much as a bf16 value's last bit.  So the
// product, its count of turns and the rest in half turns are 64-bit arithmetic (a float times an int is exact there), and sine and
// cosine are taken of a rest in [-1, 1] half turns.
#include <algorithm>
#include <cmath>

#include "paged_common.cuh"

namespace river {
namespace {

struct RopeArgs {
    Paged c;
    int layer0, n_tokens, Hq, rot;
    const void *q, *k, *v;
    int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
    const int32_t *positions, *seqs;
    const float *inv_freq;
    float scale;
    void *q_out;
    int32_t *status;
};

__device__ __forceinline__ float2 rope_turn(int pos, float inv_freq, float scale) {  // scale (cos, sin) of pos * inv_freq
    const double turns = (double)max(pos, 0) * (double)inv_freq * 0.31830988618379067154;  // in half turns
    const double rest = turns - 2.0 * rint(turns * 0.5);
    float s, c;
    sincospif((float)rest, &s, &c);
    return make_float2(c * scale, s * scale);
}
constexpr int kRopePadding = -1;  // the sequence of a token that is none
// The page of a token's place; -1: it has none (a padding token, or something is out of range, which `bad` tells).
__device__ __forceinline__ int rope_page(const RopeArgs &a, int pos, int seq, bool &bad) {
    bad = false;
    if (seq == kRopePadding) return -1;
    int page = -1;
    if (pos >= 0 && seq >= 0 && seq < a.c.n_seqs && (pos >> a.c.ps_log2) < a.c.max_pages) page = a.c.table[(size_t)seq * a.c.max_pages + (pos >> a.c.ps_log2)];
    bad = page < 0 || page >= a.c.n_pages;
    return bad ? -1 : page;
}
// Row r of a token: its query heads, its key heads, its value heads.
template <class TI, class TC>
struct RopeRow {
    const TI *src;
    TC *dst;
    bool turn;
    __device__ __forceinline__ RopeRow(const RopeArgs &a, int t, int r, int page, int inpage) {
        const int kvh = r - a.Hq;
        if (kvh < 0) {
            src = static_cast<const TI *>(a.q) + t * a.q_tok + r * a.q_head;
            dst = static_cast<TC *>(a.q_out) + ((size_t)t * a.Hq + r) * a.c.dh;
        } else {
            const bool v = kvh >= a.c.Hkv;
            const int h = v ? kvh - a.c.Hkv : kvh;
            src = v ? static_cast<const TI *>(a.v) + t * a.v_tok + h * a.v_head : static_cast<const TI *>(a.k) + t * a.k_tok + h * a.k_head;
            dst = page < 0 ? nullptr : reinterpret_cast<TC *>(a.c.pool) + a.c.row(a.layer0, page, v, h, inpage);
        }
        turn = kvh < a.c.Hkv;
    }
};

constexpr int kRopeTokens = 4;  // at most, of a CTA
// Eight values of a row, 16 or 32 bytes as they come.
template <class TI> struct Eight {
    uint4 w[sizeof(TI) / 2];
    __device__ __forceinline__ void load(const TI *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(TI) / 2; ++i) w[i] = ldg_stream16(p + i * (16 / sizeof(TI)));
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        if constexpr (sizeof(TI) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[4 * i] = __uint_as_float(w[i].x); x[4 * i + 1] = __uint_as_float(w[i].y);
                x[4 * i + 2] = __uint_as_float(w[i].z); x[4 * i + 3] = __uint_as_float(w[i].w);
            }
        } else {
            const TI *v = reinterpret_cast<const TI *>(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = to_f(v[i]);
        }
    }
};
template <class TC>
__device__ __forceinline__ void store_eight(TC *p, const float (&x)[8]) {
    uint4 w;
    TC *v = reinterpret_cast<TC *>(&w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = from_f<TC>(x[i]);
    *reinterpret_cast<uint4 *>(p) = w;
}

// Any strides and sizes: a CTA per token, a thread per pair and, for the dims that stay, per dim - or per eight of them, from the first
// multiple of eight on, where the rows allow it (`wide`).
template <class TI, class TC, bool INTER>
__global__ void __launch_bounds__(256) rope_append_any_kernel(const RopeArgs a, int wide) {
    __shared__ float2 cs[64];
    const int t = blockIdx.x, dh = a.c.dh, half = a.rot / 2, pos = a.positions[t], seq = a.seqs[t];
    for (int i = threadIdx.x; i < half; i += blockDim.x) cs[i] = rope_turn(pos, a.inv_freq[i], a.scale);
    bool bad;
    const int page = rope_page(a, pos, seq, bad), inpage = pos & ((1 << a.c.ps_log2) - 1);
    if (bad && threadIdx.x == 0) flag(a.status, RIVER_E_BADARG);
    __syncthreads();
    const int rows = a.Hq + 2 * a.c.Hkv, eights = wide ? (a.rot + 7) / 8 * 8 : dh, single = half + eights - a.rot, per = single + (dh - eights) / 8;
    for (int u = threadIdx.x; u < rows * per; u += blockDim.x) {
        const int r = u / per, i = u - r * per;
        const RopeRow<TI, TC> row(a, t, r, page, inpage);
        if (!row.dst) continue;
        if (i < half) {
            const int d0 = INTER ? 2 * i : i, d1 = INTER ? 2 * i + 1 : i + half;
            const float x = to_f(row.src[d0]), y = to_f(row.src[d1]);
            const float2 w = row.turn ? cs[i] : make_float2(1.f, 0.f);
            row.dst[d0] = from_f<TC>(seq == kRopePadding ? 0.f : row.turn ? x * w.x - y * w.y : x);
            row.dst[d1] = from_f<TC>(seq == kRopePadding ? 0.f : row.turn ? y * w.x + x * w.y : y);
        } else if (i < single) {
            row.dst[i + half] = from_f<TC>(seq == kRopePadding ? 0.f : to_f(row.src[i + half]));
        } else {
            const int d = eights + 8 * (i - single);
            Eight<TI> e;
            float p[8];
            e.load(row.src + d);
            e.get(p);
#pragma unroll
            for (int k = 0; k < 8; ++k) p[k] = seq == kRopePadding ? 0.f : p[k];
            store_eight(row.dst + d, p);
        }
    }
}

// 16-byte rows.  A CTA takes blockDim.z tokens; thread (x, y, z) unit x of the rows y, y + blockDim.y, .. of token z.  A unit is eight dims
// (interleaved: four pairs, or dims that stay), or eight pairs and their partners half a turned part further (half layout).  UNITS rows of
// a thread, 192 bytes, are under way before place and angles are known; a thread's sines and cosines are the same for all its rows.
// Prompts are bound by HBM and by the instructions beside it: 8192 tokens of 48 heads of 128, three quarters turned, bf16: 40 us without the host (41.5 with), 5.0 TB/s (44 with
// 64-bit products for every unit's address).
template <class TI, class TC, bool INTER, int UNITS>
__global__ void __launch_bounds__(256) rope_append_kernel(const RopeArgs a) {
    __shared__ float4 cs[kRopeTokens][32];  // two pairs' (cos, sin)
    const int x = threadIdx.x, y = threadIdx.y, z = threadIdx.z, ny = blockDim.y, rows = a.Hq + 2 * a.c.Hkv, half = a.rot / 2;
    const int t = blockIdx.x * blockDim.z + z;
    const bool live = t < a.n_tokens;
    // dims of this unit: d0 .. d0 + 7, and in the half layout d0 + half ..
    const bool pairs = x < (a.rot + 7) / (INTER ? 8 : 16);
    const int d0 = INTER || pairs ? 8 * x : 8 * x + half;
    const int pos = live ? a.positions[t] : 0, seq = live ? a.seqs[t] : kRopePadding;
    // this thread's units of the token's first heads, in bytes; heads are a 32-bit step apart (the launch has looked)
    const char *const q_at = static_cast<const char *>(a.q) + (t * a.q_tok + d0) * (int64_t)sizeof(TI);
    const char *const k_at = static_cast<const char *>(a.k) + (t * a.k_tok + d0) * (int64_t)sizeof(TI);
    const char *const v_at = static_cast<const char *>(a.v) + (t * a.v_tok + d0) * (int64_t)sizeof(TI) - (int64_t)a.c.Hkv * (int)a.v_head * (int)sizeof(TI);
    const int q_step = (int)a.q_head * (int)sizeof(TI), k_step = (int)a.k_head * (int)sizeof(TI), v_step = (int)a.v_head * (int)sizeof(TI), dh = a.c.dh;
    char *const q_to = static_cast<char *>(a.q_out) + ((size_t)t * a.Hq * dh + d0) * sizeof(TC);
    char *kv_to = nullptr;  // the token's place in the K half of head 0; the heads of K, then of V, follow a page's rows apart
    const int to_step = dh * (int)sizeof(TC), kv_step = to_step << a.c.ps_log2;
    float2 w[INTER ? 4 : 8];
    for (int r0 = y; r0 - y < rows; r0 += UNITS * ny) {
        Eight<TI> u[UNITS], v[INTER ? 1 : UNITS];
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            const int r = r0 + k * ny, h = r - a.Hq;
            if (!live || r >= rows) continue;
            const char *base = h < 0 ? q_at : h < a.c.Hkv ? k_at : v_at;
            const int step = h < 0 ? q_step : h < a.c.Hkv ? k_step : v_step;
            const TI *src = reinterpret_cast<const TI *>(base + (int64_t)(h < 0 ? r : h) * step);
            u[k].load(src);
            if (!INTER && pairs) v[k].load(src + half);
        }
        if (r0 == y) {
            for (int i = y * blockDim.x + x; i < half; i += blockDim.x * ny) reinterpret_cast<float2 *>(cs[z])[i] = rope_turn(pos, a.inv_freq[i], a.scale);
            bool bad;
            const int page = rope_page(a, pos, seq, bad);
            if (bad && x == 0 && y == 0) flag(a.status, RIVER_E_BADARG);
            if (page >= 0) kv_to = reinterpret_cast<char *>(a.c.pool) + (a.c.row(a.layer0, page, 0, 0, pos & ((1 << a.c.ps_log2) - 1)) + d0) * sizeof(TC);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < (INTER ? 4 : 8); e += 2) {
                const float4 c = pairs ? cs[z][(INTER ? 2 : 4) * x + e / 2] : make_float4(1.f, 0.f, 1.f, 0.f);
                w[e] = make_float2(c.x, c.y);
                w[e + 1] = make_float2(c.z, c.w);
            }
        }
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            const int r = r0 + k * ny, h = r - a.Hq;
            char *base = h < 0 ? q_to : kv_to;
            if (!live || r >= rows || !base) continue;
            TC *const dst = reinterpret_cast<TC *>(base + (int64_t)(h < 0 ? r : h) * (h < 0 ? to_step : kv_step));
            float p[8], q[8];
            u[k].get(p);
            if (!INTER && pairs) v[k].get(q);
            if (h < a.c.Hkv && pairs) {
                if constexpr (INTER) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (4 * x + e >= half) continue;  // (the last unit may be turned in part)
                        const float y0 = p[2 * e] * w[e].x - p[2 * e + 1] * w[e].y;
                        p[2 * e + 1] = p[2 * e + 1] * w[e].x + p[2 * e] * w[e].y;
                        p[2 * e] = y0;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float y0 = p[e] * w[e].x - q[e] * w[e].y;
                        q[e] = q[e] * w[e].x + p[e] * w[e].y;
                        p[e] = y0;
                    }
                }
            }
            if (seq == kRopePadding) {
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = q[e] = 0.f;
            }
            store_eight(dst, p);
            if (!INTER && pairs) store_eight(dst + half, q);
        }
    }
}

// Rows that can be taken 16 bytes at a time: addresses and strides, a token's heads within 2 GB.
bool rope_wide(const RopeArgs &a, size_t es) {
    auto ok = [&](const void *p, int64_t tok, int64_t head) { return aligned_to(p, 16) && tok * (int64_t)es % 16 == 0 && head * (int64_t)es % 16 == 0 && head < (1 << 20) && head > -(1 << 20); };
    return ok(a.q, a.q_tok, a.q_head) && ok(a.k, a.k_tok, a.k_head) && ok(a.v, a.v_tok, a.v_head);
}

template <class TI, class TC, bool INTER>
int launch_rope(const RopeArgs &a, cudaStream_t st) {
    const bool wide = rope_wide(a, sizeof(TI));
    if (!wide || (!INTER && a.rot % 16))  // (8192 tokens of 48 heads of 128, bf16, half layout, a turned part of 34: 93 us; of 128, in units, 37)
        return launch_plain(rope_append_any_kernel<TI, TC, INTER>, a.n_tokens, 256, st, a, (int)wide);
    constexpr int UNITS = (INTER ? 24 : 12) / (int)sizeof(TI);
    const int per = INTER ? a.c.dh / 8 : a.rot / 16 + (a.c.dh - a.rot) / 8, rows = a.Hq + 2 * a.c.Hkv;
    // Few tokens: a CTA each, with all the threads that its rows keep busy.  Many: CTAs of 64 threads, which take turns at fetching, turning and
    // storing (8192 tokens of 48 heads of 128, us with 64, 128, 256 threads: from fp32 49, 54, 58; interleaved bf16 39, 40, 42; half 41, 42, 40).
    const bool few = a.n_tokens < 148 * 4;
    const int most = few ? 256 : 64, y = few ? std::min(most / per, rows) : std::min(most / per, (rows + UNITS - 1) / UNITS), z = few ? 1 : std::min(std::max(1, most / (per * y)), kRopeTokens);
    return launch_plain(rope_append_kernel<TI, TC, INTER, UNITS>, (a.n_tokens + z - 1) / z, dim3(per, y, z), st, a);
}
template <class TI, class TC>
int launch_rope(const RopeArgs &a, bool inter, cudaStream_t st) {
    return inter ? launch_rope<TI, TC, true>(a, st) : launch_rope<TI, TC, false>(a, st);
}

}  // namespace
}  // namespace river

extern "C" int river_rope_frequencies(int rotary_dim, double theta, const river_rope_scaling *s, float *inv_freq, float *scale) {
    if (!inv_freq || !scale || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 4096 || !(theta > 1.0) || !std::isfinite(theta)) return RIVER_E_BADARG;
    const int kind = s ? s->kind : RIVER_ROPE_PLAIN, n = rotary_dim / 2;
    const double pi = 3.14159265358979323846;
    if (kind < RIVER_ROPE_PLAIN || kind > RIVER_ROPE_PER_PAIR) return RIVER_E_BADARG;
    if ((kind == RIVER_ROPE_LINEAR || kind == RIVER_ROPE_BY_PARTS || kind == RIVER_ROPE_RAMP) && !(s->factor > 0.0 && std::isfinite(s->factor))) return RIVER_E_BADARG;
    if ((kind == RIVER_ROPE_BY_PARTS || kind == RIVER_ROPE_RAMP) && s->original_context < 1) return RIVER_E_BADARG;
    if (kind == RIVER_ROPE_BY_PARTS && !(s->low_freq > 0.0 && s->high_freq > s->low_freq)) return RIVER_E_BADARG;
    if (kind == RIVER_ROPE_RAMP && !(s->beta_slow > 0.0 && s->beta_fast > s->beta_slow)) return RIVER_E_BADARG;
    if (kind == RIVER_ROPE_PER_PAIR) {
        if (!s->pair_factors) return RIVER_E_BADARG;
        for (int i = 0; i < n; ++i)
            if (!(s->pair_factors[i] > 0.f && std::isfinite(s->pair_factors[i]))) return RIVER_E_BADARG;
    }
    if (s && !(s->attn_scale >= 0.0 && std::isfinite(s->attn_scale))) return RIVER_E_BADARG;
    double lo = 0, hi = 0;
    if (kind == RIVER_ROPE_RAMP) {  // the pair that turns `b` times in the original context: theta^(2 i / rotary_dim) = context / (2 pi b)
        auto pair = [&](double b) { return rotary_dim * std::log(s->original_context / (b * 2 * pi)) / (2 * std::log(theta)); };
        lo = std::fmax(std::floor(pair(s->beta_fast)), 0.0);
        hi = std::fmin(std::ceil(pair(s->beta_slow)), rotary_dim - 1.0);
        if (!(hi > lo)) hi = lo + 0.001;
    }
    for (int i = 0; i < n; ++i) {
        double f = std::pow(theta, -2.0 * i / rotary_dim);
        if (kind == RIVER_ROPE_LINEAR) f /= s->factor;
        if (kind == RIVER_ROPE_PER_PAIR) f /= (double)s->pair_factors[i];
        if (kind == RIVER_ROPE_BY_PARTS) {
            const double turns = s->original_context * f / (2 * pi);
            const double keep = std::fmin(std::fmax((turns - s->low_freq) / (s->high_freq - s->low_freq), 0.0), 1.0);
            f = f * keep + f / s->factor * (1.0 - keep);
        }
        if (kind == RIVER_ROPE_RAMP) {
            const double drawn = std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
            f = f * (1.0 - drawn) + f / s->factor * drawn;
        }
        inv_freq[i] = (float)f;
    }
    *scale = s && s->attn_scale > 0.0 ? (float)s->attn_scale : kind == RIVER_ROPE_RAMP && s->factor > 1.0 ? (float)(0.1 * std::log(s->factor) + 1.0) : 1.f;
    return RIVER_OK;
}

extern "C" int river_rope_append(const river_paged *c, int layer, int n_tokens, int Hq, int in_dtype, const river_rows *q, const river_rows *k,
                                 const river_rows *v, const int32_t *positions, const int32_t *seqs, const float *inv_freq, int rotary_dim,
                                 int interleaved, float scale, void *q_out, int32_t *status, void *cuda_stream) {
    using namespace river;
    RopeArgs a;
    if (const int rc = paged_check(c, true, false, &a.c)) return rc;
    if (layer < 1 || layer > c->n_layers || n_tokens < 0 || Hq < 0 || Hq > (1 << 16) || !inv_freq || !words(inv_freq, status) || !std::isfinite(scale)) return RIVER_E_BADARG;
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > c->dh) return RIVER_E_BADARG;
    if (in_dtype != c->dtype && in_dtype != RIVER_F32) return RIVER_E_SHAPE;
    if (n_tokens == 0) return RIVER_OK;  // (rows that are none may have no address)
    const size_t es = in_dtype == RIVER_F32 ? 4 : 2;
    if (!positions || !seqs || !words(positions, seqs)) return RIVER_E_BADARG;
    if (!k || !k->p || !v || !v->p || (Hq > 0 && (!q || !q->p || !q_out)) || !aligned_to(q_out, 16)) return RIVER_E_BADARG;
    if (!aligned_to(k->p, es) || !aligned_to(v->p, es) || (Hq > 0 && !aligned_to(q->p, es))) return RIVER_E_BADARG;
    a.layer0 = layer - 1;
    a.n_tokens = n_tokens;
    a.Hq = Hq;
    a.rot = rotary_dim;
    const river_rows none = {nullptr, 0, 0}, &qr = Hq > 0 ? *q : none;
    a.q = qr.p; a.q_tok = qr.token; a.q_head = qr.head;
    a.k = k->p; a.k_tok = k->token; a.k_head = k->head;
    a.v = v->p; a.v_tok = v->token; a.v_head = v->head;
    a.positions = positions;
    a.seqs = seqs;
    a.inv_freq = inv_freq;
    a.scale = scale;
    a.q_out = q_out;
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = c->dtype == RIVER_BF16, wide = in_dtype == RIVER_F32;
    if (bf) return wide ? launch_rope<float, __nv_bfloat16>(a, interleaved != 0, st) : launch_rope<__nv_bfloat16, __nv_bfloat16>(a, interleaved != 0, st);
    return wide ? launch_rope<float, __half>(a, interleaved != 0, st) : launch_rope<__half, __half>(a, interleaved != 0, st);
}

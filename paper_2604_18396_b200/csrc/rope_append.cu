// river_rope_frequencies, river_rope_append: rotary embedding of new tokens fused with their way into the paged cache.
//
// Pair i of a head turns by a = position * inv_freq[i]:  (x, y) -> scale (x cos a - y sin a, y cos a + x sin a).  The angle is the one
// place where 32 bits do not do: at position 2^17 a float product is off by 2^-8 rad, as much as a bf16 value's last bit.  So the
// product, its count of turns and the rest in half turns are 64-bit arithmetic (a float times an int is exact there), and sine and
// cosine are taken of a rest in [-1, 1] half turns.
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

// A CTA per token; a thread per pair and, for the dims that stay, per dim.
template <class TI, class TC, bool INTER>
__global__ void __launch_bounds__(128) rope_append_kernel(const RopeArgs a) {
    __shared__ float2 cs[64];
    const int t = blockIdx.x, dh = a.c.dh, half = a.rot / 2;
    const int pos = a.positions[t], seq = a.seqs[t];
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        const double turns = (double)(pos < 0 ? 0 : pos) * (double)a.inv_freq[i] * 0.31830988618379067154;  // in half turns
        const double rest = turns - 2.0 * rint(turns * 0.5);
        float s, c;
        sincospif((float)rest, &s, &c);
        cs[i] = make_float2(c * a.scale, s * a.scale);
    }
    int page = -1;
    if (seq >= 0) {
        if (pos >= 0 && seq < a.c.n_seqs && (pos >> a.c.ps_log2) < a.c.max_pages) page = a.c.table[(size_t)seq * a.c.max_pages + (pos >> a.c.ps_log2)];
        if (page < 0 || page >= a.c.n_pages) {
            page = -1;
            if (threadIdx.x == 0) flag(a.status, RIVER_E_BADARG);
        }
    }
    const int inpage = pos & ((1 << a.c.ps_log2) - 1);
    __syncthreads();
    const int rows = a.Hq + 2 * a.c.Hkv, per = dh - half;  // a row's pairs, then the dims that stay
    for (int u = threadIdx.x; u < rows * per; u += blockDim.x) {
        const int h = u / per, i = u % per;
        const TI *src;
        TC *dst;
        bool turn = true;
        if (h < a.Hq) {
            src = static_cast<const TI *>(a.q) + t * a.q_tok + h * a.q_head;
            dst = static_cast<TC *>(a.q_out) + ((size_t)t * a.Hq + h) * dh;
        } else {
            if (page < 0) continue;
            const bool is_v = h >= a.Hq + a.c.Hkv;
            const int kvh = h - a.Hq - (is_v ? a.c.Hkv : 0);
            src = is_v ? static_cast<const TI *>(a.v) + t * a.v_tok + kvh * a.v_head : static_cast<const TI *>(a.k) + t * a.k_tok + kvh * a.k_head;
            dst = reinterpret_cast<TC *>(a.c.pool) + a.c.row(a.layer0, page, is_v, kvh, inpage);
            turn = !is_v;
        }
        if (i < half) {
            const int d0 = INTER ? 2 * i : i, d1 = INTER ? 2 * i + 1 : i + half;
            float x = to_f(src[d0]), y = to_f(src[d1]);
            if (turn) {
                const float2 w = cs[i];
                const float x1 = x * w.x - y * w.y;
                y = y * w.x + x * w.y;
                x = x1;
            }
            dst[d0] = from_f<TC>(seq < 0 ? 0.f : x);
            dst[d1] = from_f<TC>(seq < 0 ? 0.f : y);
        } else {
            const int d = i + half;
            dst[d] = from_f<TC>(seq < 0 ? 0.f : to_f(src[d]));
        }
    }
}

template <class TI, class TC>
void launch_rope(const RopeArgs &a, bool inter, cudaStream_t st) {
    if (inter) rope_append_kernel<TI, TC, true><<<a.n_tokens, 128, 0, st>>>(a);
    else rope_append_kernel<TI, TC, false><<<a.n_tokens, 128, 0, st>>>(a);
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
    if (layer < 1 || layer > c->n_layers || n_tokens < 0 || Hq < 0 || Hq > (1 << 16) || !positions || !seqs || !inv_freq || !std::isfinite(scale)) return RIVER_E_BADARG;
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > c->dh) return RIVER_E_BADARG;
    if (in_dtype != c->dtype && in_dtype != RIVER_F32) return RIVER_E_SHAPE;
    const size_t es = in_dtype == RIVER_F32 ? 4 : 2;
    if (!k || !k->p || !v || !v->p || (Hq > 0 && (!q || !q->p || !q_out)) || !aligned_to(q_out, 16)) return RIVER_E_BADARG;
    if (!aligned_to(k->p, es) || !aligned_to(v->p, es) || (Hq > 0 && !aligned_to(q->p, es))) return RIVER_E_BADARG;
    if (n_tokens == 0) return RIVER_OK;
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
    if (bf && wide) launch_rope<float, __nv_bfloat16>(a, interleaved != 0, st);
    else if (bf) launch_rope<__nv_bfloat16, __nv_bfloat16>(a, interleaved != 0, st);
    else if (wide) launch_rope<float, __half>(a, interleaved != 0, st);
    else launch_rope<__half, __half>(a, interleaved != 0, st);
    return launch_rc();
}

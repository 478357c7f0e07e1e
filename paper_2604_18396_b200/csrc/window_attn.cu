// river_window_attention: attention over a sliding window and a few first positions of a paged cache.
#include <algorithm>
#include <cmath>

#include "window_attn_step.cuh"

namespace river {
namespace {

// grid (max_q * Hq / warps, n_seqs): a warp per query row
template <class T, int DH>
__global__ void __launch_bounds__(128) window_attn_rows_kernel(const WindowArgs a) {
    const int seq = blockIdx.y, row = blockIdx.x * 4 + (threadIdx.x >> 5), i = row / a.Hq, head = row % a.Hq;
    const int t0 = a.q_start[seq], n = a.q_start[seq + 1] - t0;
    if (n < 0 || n > a.max_q || t0 < 0 || t0 + n > a.n_tokens) {
        if (threadIdx.x == 0) flag(a.status, RIVER_E_BADARG);
        return;
    }
    if (i < n) window_attn_row<T, DH>(a, t0 + i, head, seq, a.c.lens[seq] - n + i);
}

template <class T, int DH>
void launch_rows(const WindowArgs &a, cudaStream_t st) {
    window_attn_rows_kernel<T, DH><<<dim3((a.max_q * a.Hq + 3) / 4, a.c.n_seqs), 128, 0, st>>>(a);
}

template <class T, int DH>
void launch_step(const WindowArgs &a, cudaStream_t st) {
    const int splits = step_splits(a, 148);
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {(unsigned)splits, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(splits * a.c.Hkv * ((a.Hq / a.c.Hkv + 7) / 8) * a.max_q * a.c.n_seqs));
    cfg.blockDim = dim3(32 * kStepWarps);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, window_attn_step_kernel<T, DH>, a, splits);
}

template <class T, int DH>
void launch(const WindowArgs &a, cudaStream_t st) {
    if (a.max_q <= 4) launch_step<T, DH>(a, st);
    else launch_rows<T, DH>(a, st);
}

}  // namespace
}  // namespace river

extern "C" int river_window_attention(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, int Hq,
                                      const river_rows *q, int window, int sinks, float softmax_scale, void *out, int32_t *status,
                                      void *cuda_stream) {
    using namespace river;
    WindowArgs a;
    if (const int rc = paged_check(c, true, true, &a.c)) return rc;
    if (layer < 1 || layer > c->n_layers || n_tokens < 0 || max_q < 0 || !q_start || !q || !q->p || !out || window < 1 || sinks < 0) return RIVER_E_BADARG;
    if (Hq < 1 || Hq % c->Hkv || !std::isfinite(softmax_scale) || !aligned_to(out, 16)) return RIVER_E_BADARG;
    if (c->n_seqs > 65535 || Hq > 8192 || (int64_t)c->n_seqs * Hq > (1 << 26)) return RIVER_E_SHAPE;  // (the kernels' grids)
    // heads are read 16 bytes at a time
    if (!aligned_to(q->p, 16) || q->token % 8 || q->head % 8) return RIVER_E_BADARG;
    if (n_tokens == 0 || max_q == 0) return RIVER_OK;
    a.layer0 = layer - 1;
    a.n_tokens = n_tokens;
    a.max_q = max_q < n_tokens ? max_q : n_tokens;
    a.Hq = Hq;
    a.window = window;
    a.sinks = sinks;
    a.q_start = q_start;
    a.q = q->p;
    a.q_tok = q->token;
    a.q_head = q->head;
    a.scale_log2 = softmax_scale * 1.4426950408889634f;
    a.out = out;
    a.status = status;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (c->dtype == RIVER_BF16) c->dh == 64 ? launch<__nv_bfloat16, 64>(a, st) : launch<__nv_bfloat16, 128>(a, st);
    else c->dh == 64 ? launch<__half, 64>(a, st) : launch<__half, 128>(a, st);
    return launch_rc();
}

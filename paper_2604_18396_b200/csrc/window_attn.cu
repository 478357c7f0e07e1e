// river_window_attention: attention over a sliding window and a few first positions of a paged cache.
#include <algorithm>
#include <cmath>

#include "tensor_maps.h"
#include "window_attn_prompt.cuh"

namespace river {
namespace {

template <class T, int DH>
int launch_step(const WindowArgs &a, int splits, cudaStream_t st) {
    const int64_t ctas = (int64_t)splits * a.c.Hkv * ((a.Hq / a.c.Hkv + 7) / 8) * a.max_q * a.c.n_seqs;
    if (ctas > INT32_MAX) return RIVER_E_SHAPE;
    if (splits > 8 && cuda_rc(cudaFuncSetAttribute(window_attn_step_kernel<T, DH>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1))) return RIVER_E_DEVICE;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {(unsigned)splits, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(32 * kStepWarps);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = splits > 1 ? 1 : 0;
    return cuda_rc(cudaLaunchKernelEx(&cfg, window_attn_step_kernel<T, DH>, a, splits));
}

template <class T, int DH, bool SPLIT>
int launch_prompt(const PromptArgs &pa, const CUtensorMap &map, cudaStream_t st) {
    const WindowArgs &a = pa.w;
    const size_t smem = window_attn_prompt_smem();
    if (cuda_rc(cudaFuncSetAttribute(window_attn_prompt_kernel<T, DH, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem))) return RIVER_E_DEVICE;
    const int span = kWpRows / (a.Hq / a.c.Hkv) * pa.tiles;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {(unsigned)pa.splits, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.n_tokens / span + a.c.n_seqs) * a.c.Hkv * pa.splits));
    cfg.blockDim = dim3(kWpThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = SPLIT ? 1 : 0;
    return cuda_rc(cudaLaunchKernelEx(&cfg, window_attn_prompt_kernel<T, DH, SPLIT>, map, pa));
}
template <class T, int DH>
int launch_prompt(const PromptArgs &pa, cudaStream_t st) {
    const WindowArgs &a = pa.w;
    // the pages of this block, as rows of a head's dims
    CUtensorMap map;
    const size_t rows = (size_t)a.c.n_pages * 2 * a.c.Hkv << a.c.ps_log2;
    if (rows >= (1ull << 31)) return RIVER_E_SHAPE;
    if (!make_map_bf16(&map, a.c.pool + rows * DH * 2 * a.layer0, DH, rows, 16)) return RIVER_E_DEVICE;
    return pa.splits > 1 ? launch_prompt<T, DH, true>(pa, map, st) : launch_prompt<T, DH, false>(pa, map, st);
}

// Single tokens and prompts by the two estimates: a token by itself reads its window once for up to eight heads, query tiles once for
// 128 rows.  (us, single tokens / query tiles, heads of 128; 32 query and 8 KV heads, one sequence, window 4096: 2 tokens 12 / 21, 6 22
// / 22, 16 37 / 23; 64 sequences of 2: 283 / 219; window 1024, one sequence, 8 tokens 11 / 14, 16 15 / 15; 12 and 1 heads, 4 sequences of 8:
// 12 / 16.)
// Measured for windows up to 4096 and heads of 128.  Both estimates take the table's width for a sequence's length, which the host does not know, and
// that of query tiles has no bound by HBM: from windows of 32 K on, batches of single tokens of many query heads go to query tiles where they lose
// (128 rows of 1000 positions, window and table 32768: 137 us, with a table of 1024 single tokens' 103; 64 rows, 131072: 201 / 63; 128 rows of 16000,
// 32768: 1427 / 1284).  A table no wider than its sequences are long avoids that.
template <class T, int DH>
int launch(const WindowArgs &a, cudaStream_t st) {
    double step_us, prompt_us = 1e300;
    const int splits = step_splits(a, 148, step_us);
    PromptArgs pa = {a, 1, 1};
    if (a.Hq / a.c.Hkv <= kWpRows) prompt_shape(pa, 148, prompt_us);
    return step_us <= prompt_us ? launch_step<T, DH>(a, splits, st) : launch_prompt<T, DH>(pa, st);
}

// The arguments of a call, checked.  RIVER_OK with a->n_tokens or a->max_q 0: nothing is to be done.
int window_args(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, int Hq, const river_rows *q, int window, int sinks,
                float softmax_scale, void *out, int32_t *status, WindowArgs *a) {
    if (const int rc = paged_check(c, true, true, &a->c)) return rc;
    if (layer < 1 || layer > c->n_layers || n_tokens < 0 || max_q < 0 || !q_start || !words(q_start, status) || window < 1 || sinks < 0) return RIVER_E_BADARG;
    if (Hq < 1 || Hq % c->Hkv || !std::isfinite(softmax_scale)) return RIVER_E_BADARG;
    if (c->n_seqs > 65535 || Hq > 8192 || (int64_t)c->n_seqs * Hq > (1 << 26)) return RIVER_E_SHAPE;  // (the kernels' grids)
    a->layer0 = layer - 1;
    a->n_tokens = n_tokens;
    a->max_q = std::min(max_q, n_tokens);
    a->Hq = Hq;
    a->window = window;
    a->sinks = sinks;
    a->q_start = q_start;
    a->scale_log2 = softmax_scale * 1.4426950408889634f;
    a->out = out;
    a->status = status;
    if (n_tokens == 0) return RIVER_OK;  // (rows that are none may have no address)
    if (!q || !q->p || !out || !aligned_to(out, 16)) return RIVER_E_BADARG;
    // heads are read 16 bytes at a time
    if (!aligned_to(q->p, 16) || q->token % 8 || q->head % 8) return RIVER_E_BADARG;
    a->q = q->p;
    a->q_tok = q->token;
    a->q_head = q->head;
    return RIVER_OK;
}

}  // namespace
}  // namespace river

extern "C" int river_window_attention(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, int Hq,
                                      const river_rows *q, int window, int sinks, float softmax_scale, void *out, int32_t *status,
                                      void *cuda_stream) {
    using namespace river;
    WindowArgs a;
    if (const int rc = window_args(c, layer, n_tokens, max_q, q_start, Hq, q, window, sinks, softmax_scale, out, status, &a)) return rc;
    if (a.n_tokens == 0 || a.max_q == 0) return RIVER_OK;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return c->dtype == RIVER_BF16 ? (c->dh == 64 ? launch<__nv_bfloat16, 64>(a, st) : launch<__nv_bfloat16, 128>(a, st))
                                  : (c->dh == 64 ? launch<__half, 64>(a, st) : launch<__half, 128>(a, st));
}

extern "C" int river_selftest_window_timeout(const river_paged *c, int layer, int n_tokens, int max_q, const int32_t *q_start, int Hq,
                                             const river_rows *q, int window, int sinks, float softmax_scale, void *out, int32_t *status,
                                             int splits, int poll_limit, void *cuda_stream) {
    using namespace river;
    WindowArgs a;
    if (const int rc = window_args(c, layer, n_tokens, max_q, q_start, Hq, q, window, sinks, softmax_scale, out, status, &a)) return rc;
    if (a.n_tokens == 0 || a.max_q == 0 || (splits != 1 && splits != 2 && splits != 4) || poll_limit < 1 || poll_limit > (1 << 20)) return RIVER_E_BADARG;
    if (Hq / c->Hkv > kWpRows) return RIVER_E_SHAPE;
    PromptArgs pa = {a, 2, splits, (uint32_t)poll_limit, 0};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return c->dtype == RIVER_BF16 ? (c->dh == 64 ? launch_prompt<__nv_bfloat16, 64>(pa, st) : launch_prompt<__nv_bfloat16, 128>(pa, st))
                                  : (c->dh == 64 ? launch_prompt<__half, 64>(pa, st) : launch_prompt<__half, 128>(pa, st));
}

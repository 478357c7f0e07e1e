// What the operators on a caller's paged cache share (internal): the cache as kernels see it, checks of its host description, types.
#pragma once
#include <cuda_fp16.h>

#include <utility>

#include "../../include/river.h"
#include "river_common.cuh"

namespace river {

struct Paged {
    uint8_t *pool;
    const int32_t *table, *lens;
    int n_layers, n_pages, Hkv, dh, ps_log2, n_seqs, max_pages;
    // element offset of the row of position `inpage` of a page (kv: 0 K, 1 V)
    __device__ __forceinline__ size_t row(int layer0, int page, int kv, int kvh, int inpage) const {
        return ((((((size_t)layer0 * n_pages + page) * 2 + kv) * Hkv + kvh) << ps_log2) + inpage) * (size_t)dh;
    }
};

inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// int32 and float arrays (NULL is aligned)
template <class... P>
bool words(const P *...p) {
    return ((reinterpret_cast<uintptr_t>(p) | ... | 0) & 3) == 0;
}

// The description of a cache, checked (need_pool: the call touches the pool's values).  Every offset in elements fits 63 bits; page
// ids, table columns and positions fit 31.
inline int paged_check(const river_paged *c, bool need_pool, bool need_lens, Paged *o) {
    if (!c || !c->table || (need_pool && !c->pool) || (need_lens && !c->lens)) return RIVER_E_BADARG;
    if (!aligned_to(c->pool, 128) || !aligned_to(c->table, 4) || !aligned_to(c->lens, 4)) return RIVER_E_BADARG;
    if (c->n_layers < 1 || c->n_pages < 1 || c->Hkv < 1 || c->n_seqs < 1 || c->max_pages < 1) return RIVER_E_BADARG;
    if (c->dtype != RIVER_BF16 && c->dtype != RIVER_F16) return RIVER_E_SHAPE;
    if (c->dh != 64 && c->dh != 128) return RIVER_E_SHAPE;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64) return RIVER_E_SHAPE;
    if (c->Hkv > 1024 || c->n_layers > 4096 || c->n_seqs > (1 << 20)) return RIVER_E_SHAPE;
    if ((int64_t)c->max_pages * c->page_size > INT32_MAX / 2) return RIVER_E_SHAPE;  // (positions, with room for a window's arithmetic)
    const int lg = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : 6;
    *o = Paged{static_cast<uint8_t *>(c->pool), c->table, c->lens, c->n_layers, c->n_pages, c->Hkv, c->dh, lg, c->n_seqs, c->max_pages};
    return RIVER_OK;
}

// What a runtime call of this call answered.  A failure is taken out of the runtime's record, where another call would find it as its own.
inline int cuda_rc(cudaError_t e) {
    if (e == cudaSuccess) return RIVER_OK;
    cudaGetLastError();
    return RIVER_E_DEVICE;
}
// grid x block threads of a kernel, with nothing else to its launch
template <class... P, class... A>
int launch_plain(void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t st, A &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = st;
    return cuda_rc(cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...));
}

template <class T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ void flag(int32_t *status, int code) {
    if (status) atomicMin(status, code);  // (a wait that ran out, RIVER_E_TIMEOUT, is not hidden by another CTA's RIVER_E_BADARG)
}

}  // namespace river

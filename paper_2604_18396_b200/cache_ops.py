"""Operators for long contexts on a paged cache (river_rope_append, river_window_attention, river_pages_*), over torch tensors.

Argument marshalling and checks only, like binding.py: every operator is one call into the CUDA library, asynchronous on `stream`
(default: torch's current stream); there is no fallback.  A cache is

    pool   bf16 or f16 [n_layers, n_pages, 2 (K, V), Hkv, page_size, dh]   page_size 16, 32 or 64; dh 64 or 128
    table  int32 [n_seqs, max_pages]                                       page of positions page_size * j ..; -1: none
    lens   int32 [n_seqs]                                                  positions held
    refs   int32 [n_pages]                                                 table entries that hold a page; 0: free

all contiguous CUDA tensors of one device.  A context's pool (River.kv_pool) has the same layout.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from .binding import RiverError, load

RIVER_BF16, RIVER_F16, RIVER_F32 = 0, 1, 2
_TYPES = {torch.bfloat16: RIVER_BF16, torch.float16: RIVER_F16, torch.float32: RIVER_F32}
ROPE_KINDS = {"none": 0, "linear": 1, "by_parts": 2, "ramp": 3, "per_pair": 4}


class river_paged(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("table", C.c_void_p), ("lens", C.c_void_p)] + [
        (n, C.c_int32) for n in ("dtype", "n_layers", "n_pages", "Hkv", "dh", "page_size", "n_seqs", "max_pages")]


class river_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64)]


class river_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("original_context", C.c_int32)] + [
        (n, C.c_double) for n in ("factor", "low_freq", "high_freq", "beta_fast", "beta_slow", "attn_scale")] + [
        ("pair_factors", C.POINTER(C.c_float))]


def _check(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _i32(t: Optional[torch.Tensor], shape, what: str) -> int:
    if t is None:
        return 0
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{what}: a contiguous CUDA int32 tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _cache(pool: torch.Tensor, table: torch.Tensor, lens: Optional[torch.Tensor]) -> river_paged:
    _check(pool.dim() == 6 and pool.shape[2] == 2 and pool.is_cuda and pool.is_contiguous() and pool.dtype in (torch.bfloat16, torch.float16),
           "pool: a contiguous CUDA bf16 or f16 tensor [n_layers, n_pages, 2, Hkv, page_size, dh]")
    _check(table.dim() == 2, "table: [n_seqs, max_pages]")
    s = pool.shape
    return river_paged(pool.data_ptr(), _i32(table, table.shape, "table"), _i32(lens, table.shape[:1], "lens"), _TYPES[pool.dtype], s[0], s[1],
                       s[3], s[5], s[4], table.shape[0], table.shape[1])


def _rows(x: torch.Tensor, what: str) -> river_rows:
    _check(x.dim() == 3 and x.is_cuda and (x.stride(2) == 1 or x.shape[2] == 1), f"{what}: a CUDA tensor [tokens, heads, dh] with consecutive dims")
    return river_rows(x.data_ptr(), x.stride(0), x.stride(1))


def _run(device: torch.device, stream, used: Sequence[Optional[torch.Tensor]], call):
    """call(cudaStream_t) on `stream`, with the tensors' device current; memory of `used` that another stream hands out stays theirs."""
    cur = torch.cuda.current_stream(device)
    st = cur if stream is None else stream
    if device.index == torch.cuda.current_device():
        rc = call(st.cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = call(st.cuda_stream)
    if rc:
        raise RiverError(rc, "the call was refused")
    if st != cur:
        for t in used:
            if t is not None:
                t.record_stream(st)


def _same_device(device: torch.device, *ts: Optional[torch.Tensor]):
    for t in ts:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and {t.device}")


def rope_frequencies(rotary_dim: int, theta: float, kind: str = "none", *, factor: float = 1.0, original_context: int = 0, low_freq: float = 1.0,
                     high_freq: float = 4.0, beta_fast: float = 32.0, beta_slow: float = 1.0, attn_scale: float = 0.0,
                     pair_factors: Optional[Sequence[float]] = None) -> Tuple[torch.Tensor, float]:
    """river_rope_frequencies -> (CPU float32 [rotary_dim / 2] radians per position, factor on the turned values).

    kind: none, linear, by_parts, ramp, per_pair (see include/river.h); attn_scale 0 = the kind's own."""
    _check(kind in ROPE_KINDS, f"kind: one of {', '.join(ROPE_KINDS)}")
    n = max(0, rotary_dim // 2)
    _check(pair_factors is None or len(pair_factors) == n, "pair_factors: one per pair")
    pf = (C.c_float * n)(*pair_factors) if pair_factors is not None else None
    s = river_rope_scaling(ROPE_KINDS[kind], original_context, factor, low_freq, high_freq, beta_fast, beta_slow, attn_scale, pf)
    out, scale = torch.empty(n, dtype=torch.float32), C.c_float(0.0)
    rc = load().river_rope_frequencies(rotary_dim, theta, C.byref(s), out.data_ptr(), C.byref(scale))
    if rc:
        raise RiverError(rc, "river_rope_frequencies rejected the call")
    return out, scale.value


def rope_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, seqs: torch.Tensor, inv_freq: torch.Tensor,
                pool: torch.Tensor, layer: int, table: torch.Tensor, q_out: Optional[torch.Tensor], *, interleaved: bool = False,
                scale: float = 1.0, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_rope_append: turns the heads of new tokens, queries to q_out, keys and values into block `layer` (1-based) of the cache.

    q, k, v: [tokens, heads, dh] of the pool's type or float32, any strides over tokens and heads (q and q_out may be None); positions,
    seqs: int32 [tokens] (sequence -1: padding); inv_freq: float32 [rotary_dim / 2]; status: int32 [1], set where a token has no place."""
    c = _cache(pool, table, None)
    n, hkv, dh = k.shape
    _check(v.shape == k.shape and dh == c.dh and hkv == c.Hkv and k.dtype == v.dtype and k.dtype in _TYPES, "k, v: [tokens, Hkv, dh] of one type")
    _check(inv_freq.dtype == torch.float32 and inv_freq.is_cuda and inv_freq.dim() == 1 and inv_freq.is_contiguous(), "inv_freq: CUDA float32 [rotary_dim / 2]")
    _same_device(pool.device, q, k, v, positions, seqs, inv_freq, table, q_out, status)
    hq, qr, qo = 0, None, 0
    if q is not None:
        hq = q.shape[1]
        _check(q.dtype == k.dtype and q.shape == (n, hq, dh), "q: [tokens, Hq, dh] of the type of k")
        _check(q_out is not None and q_out.shape == q.shape and q_out.is_contiguous() and q_out.dtype == pool.dtype, "q_out: contiguous, q's shape, the pool's type")
        qr, qo = C.byref(_rows(q, "q")), q_out.data_ptr()
    kr, vr = _rows(k, "k"), _rows(v, "v")
    p, s, st = _i32(positions, (n,), "positions"), _i32(seqs, (n,), "seqs"), _i32(status, (1,), "status")
    _run(pool.device, stream, (q, k, v, positions, seqs, inv_freq, pool, table, q_out, status), lambda cs: load().river_rope_append(
        C.byref(c), layer, n, hq, _TYPES[k.dtype], qr, C.byref(kr), C.byref(vr), p, s, inv_freq.data_ptr(), 2 * inv_freq.shape[0],
        1 if interleaved else 0, scale, qo, st, cs))


def window_attention(q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, pool: torch.Tensor, layer: int, table: torch.Tensor,
                     lens: torch.Tensor, *, window: int, sinks: int = 0, max_q: int, softmax_scale: Optional[float] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_window_attention: out[t] = attention of q[t] over the last `window` and the first `sinks` positions of its sequence.

    q: [tokens, Hq, dh] of the pool's type (any strides over tokens and heads that are multiples of 8); sequence s has the rows q_start[s] ..
    q_start[s + 1] - 1 (int32 [n_seqs + 1]), its last positions, at most max_q of them; softmax_scale: default 1 / sqrt(dh)."""
    c = _cache(pool, table, lens)
    _check(q.dtype == pool.dtype and q.dim() == 3 and q.shape[2] == c.dh, "q: [tokens, Hq, dh] of the pool's type")
    _check(out.dtype == q.dtype and out.shape == q.shape and out.is_contiguous(), "out: contiguous, q's shape and type")
    _same_device(pool.device, q, out, q_start, table, lens, status)
    r, qs, st = _rows(q, "q"), _i32(q_start, (c.n_seqs + 1,), "q_start"), _i32(status, (1,), "status")
    sc = c.dh ** -0.5 if softmax_scale is None else softmax_scale
    _run(pool.device, stream, (q, out, q_start, pool, table, lens, status), lambda cs: load().river_window_attention(
        C.byref(c), layer, q.shape[0], max_q, qs, q.shape[1], C.byref(r), window, sinks, sc, out.data_ptr(), st, cs))


def pages_advance(table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, n_new: torch.Tensor, table_out: torch.Tensor,
                  lens_out: torch.Tensor, refs_out: torch.Tensor, status: torch.Tensor, *, page_size: int, window: int = 0, sinks: int = 0,
                  stream=None) -> None:
    """river_pages_advance: gives back the pages that window and sinks no longer need, hands out those of n_new[s] more positions.

    The outputs may be the inputs.  status (int32 [1]): 0, -4 (not enough pages: nothing was handed out) or -1."""
    _check(table.dim() == 2 and refs.dim() == 1, "table: [n_seqs, max_pages], refs: [n_pages]")
    s = table.shape
    c = river_paged(0, _i32(table, s, "table"), _i32(lens, s[:1], "lens"), RIVER_BF16, 1, refs.shape[0], 1, 64, page_size, s[0], s[1])
    a = (_i32(refs, refs.shape, "refs"), _i32(n_new, s[:1], "n_new"), window, sinks, _i32(table_out, s, "table_out"), _i32(lens_out, s[:1], "lens_out"),
         _i32(refs_out, refs.shape, "refs_out"), _i32(status, (1,), "status"))
    ts = (table, lens, refs, n_new, table_out, lens_out, refs_out, status)
    _same_device(table.device, *ts)
    _run(table.device, stream, ts, lambda cs: load().river_pages_advance(C.byref(c), *a, cs))


def pages_reorder(pool: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, parents: torch.Tensor,
                  table_out: torch.Tensor, lens_out: torch.Tensor, refs_out: torch.Tensor, status: torch.Tensor, *,
                  copies: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_pages_reorder: sequence i becomes what sequence parents[i] was (-1: empty); whole pages are shared, last pages copied.

    The outputs overlap no input.  copies (int32 [1 + 3 n_seqs]): the pages that were copied, for callers who want to know."""
    c = _cache(pool, table, lens)
    s = table.shape
    if copies is None:
        copies = torch.empty(1 + 3 * s[0], dtype=torch.int32, device=table.device)
    a = (_i32(refs, (c.n_pages,), "refs"), _i32(parents, s[:1], "parents"), _i32(table_out, s, "table_out"), _i32(lens_out, s[:1], "lens_out"),
         _i32(refs_out, refs.shape, "refs_out"), _i32(copies, (1 + 3 * s[0],), "copies"), _i32(status, (1,), "status"))
    ts = (pool, table, lens, refs, parents, table_out, lens_out, refs_out, copies, status)
    _same_device(pool.device, *ts)
    _run(pool.device, stream, ts, lambda cs: load().river_pages_reorder(C.byref(c), *a, cs))


def pages_compact(pool: torch.Tensor, table: torch.Tensor, refs: torch.Tensor, table_out: torch.Tensor, refs_out: torch.Tensor,
                  remap: torch.Tensor, n_used: torch.Tensor, *, moves: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_pages_compact: the pages in use move to the lowest ids; remap[p]: where page p went (-1: free).

    table_out and refs_out may be the inputs.  moves (int32 [1 + n_pages]): which pages moved, for callers who want to know."""
    c = _cache(pool, table, None)
    n = (c.n_pages,)
    if moves is None:
        moves = torch.empty(1 + c.n_pages, dtype=torch.int32, device=table.device)
    a = (_i32(refs, n, "refs"), _i32(table_out, table.shape, "table_out"), _i32(refs_out, n, "refs_out"), _i32(remap, n, "remap"),
         _i32(n_used, (1,), "n_used"), _i32(moves, (1 + c.n_pages,), "moves"))
    ts = (pool, table, refs, table_out, refs_out, remap, n_used, moves)
    _same_device(pool.device, *ts)
    _run(pool.device, stream, ts, lambda cs: load().river_pages_compact(C.byref(c), *a, cs))

"""Operators on a paged cache, for long contexts and for requests that share prefixes (river_rope_append, river_window_attention, river_prefix_*,
river_pages_*), over torch tensors.

Argument marshalling and checks only, like binding.py: every operator is one call into the CUDA library, asynchronous on `stream`
(default: torch's current stream; another one has been ordered behind the inputs' by the caller); there is no fallback.  A cache is

    pool   bf16 or f16 [n_layers, n_pages, 2 (K, V), Hkv, page_size, dh]   page_size 16, 32 or 64; dh 64 or 128
    table  int32 [n_seqs, max_pages]                                       page of positions page_size * j ..; -1: none
    lens   int32 [n_seqs]                                                  positions held
    refs   int32 [n_pages]                                                 table entries that hold a page; 0: free

all contiguous CUDA tensors of one device.  status (int32 [1]) takes what only the device can see: rope_append, window_attention, prefix_attention and
pages_slots write it only where something is wrong (the lowest code stays), pages_advance, pages_reorder and pages_admit every time - so not one word for
both.  A context's pool (River.kv_pool) is not for them: its page table stays with the context.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Sequence, Tuple

import torch

from .binding import RiverError, load

RIVER_BF16, RIVER_F16, RIVER_F32 = 0, 1, 2
_BF16, _F16, _F32, _I32 = torch.bfloat16, torch.float16, torch.float32, torch.int32
_TYPES = {_BF16: RIVER_BF16, _F16: RIVER_F16, _F32: RIVER_F32}
ROPE_KINDS = {"none": 0, "linear": 1, "by_parts": 2, "ramp": 3, "per_pair": 4}
# A call takes 5 to 9 us of host time, half of it the launch itself: the structs go as packed bytes (river_paged and river_rows below are their
# layouts), devices are compared as numbers, and the stream comes as the pointer that torch keeps.
_PAGED, _ROWS = struct.Struct("@PPP8i"), struct.Struct("@Pqq")


class river_paged(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("table", C.c_void_p), ("lens", C.c_void_p)] + [
        (n, C.c_int32) for n in ("dtype", "n_layers", "n_pages", "Hkv", "dh", "page_size", "n_seqs", "max_pages")]


class river_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64)]


class river_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("original_context", C.c_int32)] + [
        (n, C.c_double) for n in ("factor", "low_freq", "high_freq", "beta_fast", "beta_slow", "attn_scale")] + [
        ("pair_factors", C.POINTER(C.c_float))]


def _refuse(what: str):
    raise ValueError(what)


def _ints(bits: int, what: str):
    """`bits`: numbers or'ed together; ctypes would cut off what 32 bits do not hold (a negative one among them is refused by the library)."""
    if not -0x80000000 <= bits <= 0x7fffffff:
        _refuse(f"{what}: numbers of 32 bits")


def _i32(t: torch.Tensor, shape, device: int, what: str) -> int:
    if t.dtype is not _I32 or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _refuse(f"{what}: a contiguous int32 tensor of shape {tuple(shape)} on CUDA device {device}")
    return t.data_ptr()


def _cache(pool: torch.Tensor, table: torch.Tensor, lens: Optional[torch.Tensor], device: int) -> bytes:
    s, ts = pool.shape, table.shape
    if len(s) != 6 or s[2] != 2 or device < 0 or not pool.is_contiguous() or pool.dtype not in (_BF16, _F16):
        _refuse("pool: a contiguous CUDA bf16 or f16 tensor [n_layers, n_pages, 2, Hkv, page_size, dh]")
    if len(ts) != 2:
        _refuse("table: [n_seqs, max_pages]")
    return _PAGED.pack(pool.data_ptr(), _i32(table, ts, device, "table"), _i32(lens, ts[:1], device, "lens") if lens is not None else 0,
                       _TYPES[pool.dtype], s[0], s[1], s[3], s[5], s[4], ts[0], ts[1])


def _rows(x: torch.Tensor, device: int, what: str) -> bytes:
    t, h, d = x.stride()
    if x.get_device() != device or (d != 1 and x.shape[2] != 1):
        _refuse(f"{what}: a tensor [tokens, heads, dh] with consecutive dims on CUDA device {device}")
    if (t | h) & 7:  # (the step of a dim with one place may be anything, and only an odd one would be in the way)
        t, h = t if x.shape[0] > 1 else 0, h if x.shape[1] > 1 else 0
    return _ROWS.pack(x.data_ptr(), t, h)


def _run(fn, device: int, stream, used: Sequence[Optional[torch.Tensor]], *args):
    """fn(*args, cudaStream_t) on `stream`, with the tensors' device current; memory of `used` that another stream hands out stays theirs."""
    cur = torch._C._cuda_getCurrentRawStream(device)
    st = cur if stream is None else stream.cuda_stream
    if device == torch._C._cuda_getDevice():
        rc = fn(*args, st)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, st)
    if rc:
        raise RiverError(rc, f"{fn.__name__} refused the call")
    if st != cur:
        for t in used:
            if t is not None:
                t.record_stream(stream)


def _scratch(n: int, device: torch.device, stream) -> torch.Tensor:
    """n ints from the memory of the stream that uses them (what another stream hands out may be in use there still)."""
    if stream is None:
        return torch.empty(n, dtype=_I32, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=_I32, device=device)


def rope_frequencies(rotary_dim: int, theta: float, kind: str = "none", *, factor: float = 1.0, original_context: int = 0, low_freq: float = 1.0,
                     high_freq: float = 4.0, beta_fast: float = 32.0, beta_slow: float = 1.0, attn_scale: float = 0.0,
                     pair_factors: Optional[Sequence[float]] = None) -> Tuple[torch.Tensor, float]:
    """river_rope_frequencies -> (CPU float32 [rotary_dim / 2] radians per position, factor on the turned values).

    kind: none, linear, by_parts, ramp, per_pair (see include/river.h); attn_scale 0 = the kind's own."""
    _ints(rotary_dim | original_context, "rotary_dim, original_context")
    n = max(0, rotary_dim // 2)
    if kind not in ROPE_KINDS:
        _refuse(f"kind: one of {', '.join(ROPE_KINDS)}")
    if pair_factors is not None and len(pair_factors) != n:
        _refuse("pair_factors: one per pair")
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
    _ints(layer, "layer")
    dev = pool.get_device()
    c = _cache(pool, table, None, dev)
    n, hkv, dh = k.shape
    dt = k.dtype
    if v.shape != k.shape or dh != pool.shape[5] or hkv != pool.shape[3] or v.dtype is not dt or dt not in _TYPES:
        _refuse("k, v: [tokens, Hkv, dh] of one type")
    if inv_freq.dtype is not _F32 or inv_freq.dim() != 1 or inv_freq.get_device() != dev or not inv_freq.is_contiguous():
        _refuse("inv_freq: CUDA float32 [rotary_dim / 2]")
    hq, qr, qo = 0, None, 0
    if q is not None:
        hq = q.shape[1]
        if q.dtype is not dt or q.shape != (n, hq, dh):
            _refuse("q: [tokens, Hq, dh] of the type of k")
        if q_out is None or q_out.shape != q.shape or q_out.get_device() != dev or not q_out.is_contiguous() or q_out.dtype is not pool.dtype:
            _refuse("q_out: contiguous, q's shape, the pool's type")
        qr, qo = _rows(q, dev, "q"), q_out.data_ptr()
    _run(load().river_rope_append, dev, stream, (q, k, v, positions, seqs, inv_freq, pool, table, q_out, status), c, layer, n, hq, _TYPES[dt], qr,
         _rows(k, dev, "k"), _rows(v, dev, "v"), _i32(positions, (n,), dev, "positions"), _i32(seqs, (n,), dev, "seqs"), inv_freq.data_ptr(),
         2 * inv_freq.shape[0], 1 if interleaved else 0, scale, qo, 0 if status is None else _i32(status, (1,), dev, "status"))


def window_attention(q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, pool: torch.Tensor, layer: int, table: torch.Tensor,
                     lens: torch.Tensor, *, window: int, sinks: int = 0, max_q: int, softmax_scale: Optional[float] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_window_attention: out[t] = attention of q[t] over the last `window` and the first `sinks` positions of its sequence.

    q: [tokens, Hq, dh] of the pool's type (any strides over tokens and heads that are multiples of 8); sequence s has the rows q_start[s] ..
    q_start[s + 1] - 1 (int32 [n_seqs + 1]), its last positions, at most max_q of them; softmax_scale: default 1 / sqrt(dh)."""
    _ints(layer | window | sinks | max_q, "layer, window, sinks, max_q")
    dev, qs = pool.get_device(), q.shape
    c = _cache(pool, table, lens, dev)
    if q.dtype is not pool.dtype or len(qs) != 3 or qs[2] != pool.shape[5]:
        _refuse("q: [tokens, Hq, dh] of the pool's type")
    if out.dtype is not q.dtype or out.shape != qs or out.get_device() != dev or not out.is_contiguous():
        _refuse("out: contiguous, q's shape and type")
    _run(load().river_window_attention, dev, stream, (q, out, q_start, pool, table, lens, status), c, layer, qs[0], max_q,
         _i32(q_start, (table.shape[0] + 1,), dev, "q_start"), qs[1], _rows(q, dev, "q"), window, sinks,
         qs[2] ** -0.5 if softmax_scale is None else softmax_scale, out.data_ptr(), 0 if status is None else _i32(status, (1,), dev, "status"))


def pages_advance(table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, n_new: torch.Tensor, table_out: torch.Tensor,
                  lens_out: torch.Tensor, refs_out: torch.Tensor, status: torch.Tensor, *, page_size: int, window: int = 0, sinks: int = 0,
                  stream=None) -> None:
    """river_pages_advance: gives back the pages that window and sinks no longer need, hands out those of n_new[s] more positions.

    The outputs may be the inputs.  status (int32 [1]): 0, -4 (not enough pages: nothing was handed out) or -1."""
    _ints(page_size | window | sinks, "page_size, window, sinks")
    dev, s, r = table.get_device(), table.shape, refs.shape
    if len(s) != 2 or len(r) != 1 or dev < 0:
        _refuse("table: [n_seqs, max_pages], refs: [n_pages], CUDA tensors")
    n = s[:1]
    c = _PAGED.pack(0, _i32(table, s, dev, "table"), _i32(lens, n, dev, "lens"), RIVER_BF16, 1, r[0], 1, 64, page_size, s[0], s[1])
    _run(load().river_pages_advance, dev, stream, (table, lens, refs, n_new, table_out, lens_out, refs_out, status), c, _i32(refs, r, dev, "refs"),
         _i32(n_new, n, dev, "n_new"), window, sinks, _i32(table_out, s, dev, "table_out"), _i32(lens_out, n, dev, "lens_out"),
         _i32(refs_out, r, dev, "refs_out"), _i32(status, (1,), dev, "status"))


def pages_reorder(pool: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, parents: torch.Tensor,
                  table_out: torch.Tensor, lens_out: torch.Tensor, refs_out: torch.Tensor, status: torch.Tensor, *,
                  copies: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_pages_reorder: sequence i becomes what sequence parents[i] was (-1: empty); whole pages are shared, last pages copied.

    The outputs overlap no input.  copies (int32 [1 + 3 n_seqs]): the pages that were copied, for callers who want to know."""
    dev, s = pool.get_device(), table.shape
    c = _cache(pool, table, lens, dev)
    n, r = s[:1], pool.shape[1:2]
    if copies is None:
        copies = _scratch(1 + 3 * s[0], pool.device, stream)
    _run(load().river_pages_reorder, dev, stream, (pool, table, lens, refs, parents, table_out, lens_out, refs_out, copies, status), c,
         _i32(refs, r, dev, "refs"), _i32(parents, n, dev, "parents"), _i32(table_out, s, dev, "table_out"), _i32(lens_out, n, dev, "lens_out"),
         _i32(refs_out, r, dev, "refs_out"), _i32(copies, (1 + 3 * s[0],), dev, "copies"), _i32(status, (1,), dev, "status"))


def pages_compact(pool: torch.Tensor, table: torch.Tensor, refs: torch.Tensor, table_out: torch.Tensor, refs_out: torch.Tensor,
                  remap: torch.Tensor, n_used: torch.Tensor, *, moves: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_pages_compact: the pages in use move to the lowest ids; remap[p]: where page p went (-1: free).

    table_out and refs_out may be the inputs.  moves (int32 [1 + n_pages]): which pages moved, for callers who want to know."""
    dev, s = pool.get_device(), table.shape
    c = _cache(pool, table, None, dev)
    r = pool.shape[1:2]
    if moves is None:
        moves = _scratch(1 + r[0], pool.device, stream)
    _run(load().river_pages_compact, dev, stream, (pool, table, refs, table_out, refs_out, remap, n_used, moves), c, _i32(refs, r, dev, "refs"),
         _i32(table_out, s, dev, "table_out"), _i32(refs_out, r, dev, "refs_out"), _i32(remap, r, dev, "remap"), _i32(n_used, (1,), dev, "n_used"),
         _i32(moves, (1 + r[0],), dev, "moves"))


def _table(table: torch.Tensor, lens: torch.Tensor, n_pages: int, page_size: int, device: int) -> bytes:
    """A cache of which a call touches the page table only."""
    s = table.shape
    if len(s) != 2 or device < 0:
        _refuse("table: [n_seqs, max_pages], a CUDA tensor")
    return _PAGED.pack(0, _i32(table, s, device, "table"), _i32(lens, s[:1], device, "lens"), RIVER_BF16, 1, n_pages, 1, 64, page_size, s[0], s[1])


def pages_admit(table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, like: torch.Tensor, begin: torch.Tensor, total: torch.Tensor,
                table_out: torch.Tensor, lens_out: torch.Tensor, refs_out: torch.Tensor, n_new: torch.Tensor, status: torch.Tensor, *,
                page_size: int, stream=None) -> None:
    """river_pages_admit: sequence i becomes a request of total[i] positions that begins with the first begin[i] of what sequence like[i] was (-1:
    none; i: it goes on); whole pages are shared, the others the lowest free ones.

    The outputs overlap no input.  n_new (int32 [n_seqs]): positions that are still to be computed; status (int32 [1]): 0, -4 (not enough pages: the
    state as it was) or -1."""
    _ints(page_size, "page_size")
    dev, s, r = table.get_device(), table.shape, refs.shape
    if len(r) != 1:
        _refuse("refs: [n_pages]")
    c = _table(table, lens, r[0], page_size, dev)
    n = s[:1]
    _run(load().river_pages_admit, dev, stream, (table, lens, refs, like, begin, total, table_out, lens_out, refs_out, n_new, status), c,
         _i32(refs, r, dev, "refs"), _i32(like, n, dev, "like"), _i32(begin, n, dev, "begin"), _i32(total, n, dev, "total"),
         _i32(table_out, s, dev, "table_out"), _i32(lens_out, n, dev, "lens_out"), _i32(refs_out, r, dev, "refs_out"), _i32(n_new, n, dev, "n_new"),
         _i32(status, (1,), dev, "status"))


def pages_slots(table: torch.Tensor, lens: torch.Tensor, n_new: torch.Tensor, q_start: torch.Tensor, positions: torch.Tensor, seqs: torch.Tensor,
                slots: torch.Tensor, *, page_size: int, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_pages_slots: where the last n_new[s] positions of each sequence stand, row by row.

    q_start: int32 [n_seqs + 1]; positions, seqs: int32 [tokens]; slots: int64 [tokens], page * page_size + place in the page.  Rows behind the
    last sequence's are -1 (padding, as rope_append has it)."""
    _ints(page_size, "page_size")
    dev = table.get_device()
    c = _table(table, lens, 1, page_size, dev)
    t = positions.shape
    if len(t) != 1:
        _refuse("positions: [tokens]")
    if slots.dtype is not torch.int64 or slots.get_device() != dev or slots.shape != t or not slots.is_contiguous():
        _refuse(f"slots: a contiguous int64 tensor of shape {tuple(t)} on CUDA device {dev}")
    _run(load().river_pages_slots, dev, stream, (table, lens, n_new, q_start, positions, seqs, slots, status), c, _i32(n_new, lens.shape, dev, "n_new"), t[0],
         _i32(q_start, (table.shape[0] + 1,), dev, "q_start"), _i32(positions, t, dev, "positions"), _i32(seqs, t, dev, "seqs"), slots.data_ptr(),
         0 if status is None else _i32(status, (1,), dev, "status"))


def prefix_groups(table: torch.Tensor, lens: torch.Tensor, q_start: torch.Tensor, lead: torch.Tensor, shared: torch.Tensor, *, page_size: int,
                  least: int = 1, stream=None) -> None:
    """river_prefix_groups: lead[s] = the first sequence of the group that s shares its first pages with, shared[s] = how many positions.

    Groups are neighbours that share `least` positions or more before their new tokens, of which sequence s has q_start[s + 1] - q_start[s].  A group shares
    what all of its neighbours do: `least` is above what all requests begin with, where some share more."""
    _ints(page_size | least, "page_size, least")
    dev = table.get_device()
    c = _table(table, lens, 1, page_size, dev)
    _run(load().river_prefix_groups, dev, stream, (table, lens, q_start, lead, shared), c, _i32(q_start, (table.shape[0] + 1,), dev, "q_start"), least,
         _i32(lead, lens.shape, dev, "lead"), _i32(shared, lens.shape, dev, "shared"))


def prefix_attention(q: torch.Tensor, out: torch.Tensor, q_start: torch.Tensor, pool: torch.Tensor, layer: int, table: torch.Tensor, lens: torch.Tensor,
                     lead: torch.Tensor, shared: torch.Tensor, *, max_q: int, max_own: int = 0, softmax_scale: Optional[float] = None,
                     workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """river_prefix_attention: out[t] = causal attention of q[t] over its sequence, whose first shared[s] positions the group of lead[s] holds in the same
    pages; they are read once for all of it where that is expected to take less time.

    q: [tokens, Hq, dh] of the pool's type (any strides over tokens and heads that are multiples of 8); sequence s has the rows q_start[s] ..
    q_start[s + 1] - 1 (int32 [n_seqs + 1]), its last positions, at most max_q of them; max_own: about the most positions behind the shared ones (0: not
    known; by that and the table's width the way of computing is chosen: both are best near what the sequences hold); softmax_scale: default 1 / sqrt(dh); workspace (uint8): for callers who keep one,
    prefix_attention_bytes of them; calls that may run at the same time have one each."""
    _ints(layer | max_q | max_own, "layer, max_q, max_own")
    dev, qs, n = pool.get_device(), q.shape, lens.shape
    c = _cache(pool, table, lens, dev)
    if q.dtype is not pool.dtype or len(qs) != 3 or qs[2] != pool.shape[5]:
        _refuse("q: [tokens, Hq, dh] of the pool's type")
    if out.dtype is not q.dtype or out.shape != qs or out.get_device() != dev or not out.is_contiguous():
        _refuse("out: contiguous, q's shape and type")
    if workspace is not None and (workspace.dtype is not torch.uint8 or workspace.dim() != 1 or workspace.get_device() != dev or not workspace.is_contiguous()):
        _refuse("workspace: contiguous CUDA uint8 [bytes]")
    args = (c, layer, qs[0], max_q, max_own, _i32(q_start, (table.shape[0] + 1,), dev, "q_start"), _i32(lead, n, dev, "lead"), _i32(shared, n, dev, "shared"),
            qs[1], _rows(q, dev, "q"), qs[2] ** -0.5 if softmax_scale is None else softmax_scale, out.data_ptr())
    word = 0 if status is None else _i32(status, (1,), dev, "status")
    fn, used = load().river_prefix_attention, (q, out, q_start, pool, table, lens, lead, shared, workspace, status)
    if workspace is None:
        try:  # (a small call needs none, and asking the allocator takes as long as the rest of the call)
            return _run(fn, dev, stream, used, *args, 0, 0, word)
        except RiverError as e:
            if e.code != -3:
                raise
        workspace = _scratch(-(-load().river_prefix_attention_needs(c, qs[0], max_q, max_own, qs[1]) // 4), pool.device, stream)
        used = (*used[:8], workspace, status)
    _run(fn, dev, stream, used, *args, workspace.data_ptr(), workspace.nbytes, word)


def prefix_attention_bytes(n_seqs: int, tokens: int, hq: int, hkv: int, dh: int) -> int:
    """river_prefix_attention_bytes: of a workspace for every call of prefix_attention with at most that many sequences and tokens."""
    _ints(n_seqs | tokens | hq | hkv | dh, "n_seqs, tokens, heads, dh")
    return load().river_prefix_attention_bytes(n_seqs, tokens, hq, hkv, dh)

"""Python binding of the paged cache and the beams in include/dasc/cache.h (argument marshalling only).

As in ops.py: each function has the name of its C entry point and turns torch tensors into
pointers, sizes and strides; errors raise DascError.  Tensors are checked for type, shape and
device, which has to be the current one, and that every row the kernels address lies inside them.
"""

from __future__ import annotations

import ctypes as C
import struct

import torch

from . import _lib
from ._lib import LIB
from .dasc import _check, _dev, _stream
from .ops import DTYPE, _BF16, _F32, _I32, _rows, _scratch

_F16, _I64 = torch.float16, torch.int64

# The structs are packed as bytes in one step (their ctypes classes in _lib.py give the layout)
_KV_CACHE = struct.Struct("@2P7q4i")
_APPEND_IO = struct.Struct("@8P11q4i")
_ATTN_IO = struct.Struct("@6P8q7if")
assert (_KV_CACHE.size == C.sizeof(_lib.KvCache) and _APPEND_IO.size == C.sizeof(_lib.AppendIo)
        and _ATTN_IO.size == C.sizeof(_lib.AttnIo))


def _here(stream, *tensors) -> None:
    """All tensors, and the stream if one is given, on the current device: a launch goes there."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"the stream is on {stream.device}, the current device is cuda:{dev}")


def _cache(k, v):
    """(packed struct, dtype, heads, head_dim) of a layer's pages [n_pages, page_size, heads, head_dim]."""
    for t, name in ((k, "k_cache"), (v, "v_cache")):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
    dt, shape = k.dtype, k.shape
    if dt is not _BF16 and dt is not _F16:
        raise TypeError(f"k_cache must be bfloat16 or float16, got {dt}")
    if v.dtype is not dt:
        raise TypeError(f"v_cache must be {dt}, got {v.dtype}")
    if len(shape) != 4 or v.shape != shape:
        raise ValueError(f"k_cache and v_cache must be [n_pages, page_size, n_kv_heads, head_dim], got "
                         f"{list(shape)} and {list(v.shape)}")
    ks, vs = k.stride(), v.stride()
    if ks[3] != 1 or vs[3] != 1:
        raise ValueError("the last dimension of k_cache and v_cache must be contiguous")
    pages, size, heads, d = shape
    return (_KV_CACHE.pack(k.data_ptr(), v.data_ptr(), *ks[:3], *vs[:3], pages, size, heads, d, DTYPE[dt]), dt,
            heads, d)


def _list(t, dtype, n: int, name: str):
    """Pointer of a contiguous tensor of n elements."""
    p = _dev(t, dtype, name)
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements, got {t.numel()}")
    return p


def dasc_cache_append(k_cache, v_cache, slots, k, v, q=None, q_out=None, pos=None, inv_freq=None, pair_axis=None,
                      adjacent: bool = False, stream=None) -> None:
    """Rotates queries and keys by their positions and writes keys and values to their slots.

    k_cache, v_cache [n_pages, page_size, n_kv_heads, head_dim] bfloat16 or float16, in any order of
    memory but for the last dimension; slots [n_tokens] int64, page * page_size + place, outside
    the cache (-1): not stored.  k, v [n_tokens, n_kv_heads, head_dim], q and q_out [n_tokens,
    n_q_heads, head_dim] (both or neither; q_out may be q) in the cache's type, strided but for the
    last dimension.  inv_freq [rot / 2] float32 (None: no rotation) turns the first rot elements of
    each head by pos [n_tokens] or [n_tokens, n_axes] int32, pair i by the axis pair_axis[i] (int32,
    None: 0); pairs are (i, i + rot / 2), or (2 i, 2 i + 1) if adjacent.
    """
    cache, dt, heads, d = _cache(k_cache, v_cache)
    n = k.shape[0]
    pk, k0, k1 = _rows(k, dt, (n, heads, d), "k")
    pv, v0, v1 = _rows(v, dt, (n, heads, d), "v")
    ps = _list(slots, _I64, n, "slots")
    pq = pqo = pp = pf = pa = q0 = q1 = qo0 = qo1 = p0 = p1 = rot = hq = 0
    axes = 1
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if q is not None:
        hq = q.shape[1]
        pq, q0, q1 = _rows(q, dt, (n, hq, d), "q")
        pqo, qo0, qo1 = _rows(q_out, dt, (n, hq, d), "q_out")
    if (inv_freq is None) != (pos is None):
        raise ValueError("pos and inv_freq go together")
    if inv_freq is not None:
        pf, rot = _dev(inv_freq, _F32, "inv_freq"), 2 * inv_freq.numel()
        axes = 1 if pos.dim() == 1 else pos.shape[1]
        pp, p0, p1 = _rows(pos if pos.dim() == 2 else pos[:, None], _I32, (n, axes), "pos", False)
        if pair_axis is not None:
            pa = _list(pair_axis, _I32, rot // 2, "pair_axis")
    _here(stream, k_cache, v_cache, slots, k, v, q, q_out, pos, inv_freq, pair_axis)
    io = _APPEND_IO.pack(pq, pqo, pk, pv, ps, pp, pf, pa, q0, q1, qo0, qo1, k0, k1, v0, v1, p0, p1, n, hq, axes, rot,
                         adjacent)
    _check(LIB.dasc_cache_append(cache, io, _stream(stream)), "dasc_cache_append")


def dasc_cache_attn_workspace_bytes(n_req: int, n_tokens: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                                    max_len: int, max_kv: int) -> int:
    out = C.c_size_t()
    _check(LIB.dasc_cache_attn_workspace_bytes(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_len, max_kv,
                                               C.byref(out)), "dasc_cache_attn_workspace_bytes")
    return out.value


def dasc_cache_attn(k_cache, v_cache, block_table, kv_lens, q, o, cu_seqlens, max_len: int, max_kv: int | None = None,
                    scale: float | None = None, causal: bool = True, window: int = 0, lse=None, workspace=None,
                    stream=None) -> None:
    """Attention of every request's new tokens over its pages of the cache.

    q and the output o [n_tokens, n_q_heads, head_dim] in the cache's type, strided but for the last
    dimension; query head h reads key head h // (n_q_heads / n_kv_heads).  cu_seqlens [n_req + 1]
    int32 gives each request's rows, kv_lens [n_req] int32 its positions with the new tokens among
    them, already appended, block_table [n_req, width] int32 its pages.  Token j of a request's n stands at
    kv_lens - n + j and sees the positions up to its own (causal; all otherwise), the last `window`
    of them if that is not 0.  max_len and max_kv: the longest request's new tokens and positions, as
    the caller knows them (None: the table's).  scale: None is head_dim ** -0.5.  lse [n_tokens,
    n_q_heads] float32 receives the log-sums of the scores' exponentials.
    """
    cache, dt, heads, d = _cache(k_cache, v_cache)
    n, hq = q.shape[0], q.shape[1]
    n_req = cu_seqlens.numel() - 1
    pq, q0, q1 = _rows(q, dt, (n, hq, d), "q")
    po, o0, o1 = _rows(o, dt, (n, hq, d), "o")
    pl = l0 = l1 = 0
    if lse is not None:
        pl, l0, l1 = _rows(lse, _F32, (n, hq), "lse", False)
    pc = _dev(cu_seqlens, _I32, "cu_seqlens")
    pkv = _list(kv_lens, _I32, n_req, "kv_lens")
    width = block_table.shape[1]
    pt, t0, _ = _rows(block_table, _I32, (n_req, width), "block_table")
    most = width * k_cache.shape[1]
    max_kv = most if max_kv is None or max_kv > most else max_kv
    _here(stream, k_cache, v_cache, block_table, kv_lens, q, o, cu_seqlens, lse, workspace)
    need = (0 if workspace is not None else
            dasc_cache_attn_workspace_bytes(n_req, n, hq, heads, d, max_len, max_kv))
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, q.device if need else None, stream)
    io = _ATTN_IO.pack(pq, po, pl, pt, pc, pkv, q0, q1, o0, o1, l0, l1, t0, n, n_req, hq, width, max_len, max_kv,
                       causal, window, d ** -0.5 if scale is None else scale)
    _check(LIB.dasc_cache_attn(cache, io, ws_ptr, ws_bytes, _stream(stream)), "dasc_cache_attn")
    del ws


def dasc_beam_select_workspace_bytes(n_req: int, beams: int, vocab: int, n_out: int) -> int:
    out = C.c_size_t()
    _check(LIB.dasc_beam_select_workspace_bytes(n_req, beams, vocab, n_out, C.byref(out)),
           "dasc_beam_select_workspace_bytes")
    return out.value


def dasc_beam_select(logits, scores, out_scores, out_tokens, out_parents, slots=None, out_slots=None, workspace=None,
                     stream=None) -> None:
    """The best continuations over beams and vocabulary (see dasc/cache.h for the exact rule).

    logits [n_req, beams, vocab] in bfloat16, float16 or float32, rows contiguous; scores [n_req,
    beams] float32, -inf for a beam that is not in use.  Writes out_scores float32, out_tokens and
    out_parents int32 [n_req, n_out], best first; with slots [n_req, beams] int32 also out_slots, the
    slots of the parents.
    """
    if not isinstance(logits, torch.Tensor) or logits.dtype not in DTYPE:
        raise TypeError("logits must be a bfloat16, float16 or float32 tensor")
    if logits.dim() != 3 or out_scores.dim() != 2:
        raise ValueError("logits must be [n_req, beams, vocab], out_scores [n_req, n_out]")
    n, beams, vocab = logits.shape
    n_out = out_scores.shape[1]
    px, x0, x1 = _rows(logits, logits.dtype, (n, beams, vocab), "logits")
    pc = _list(scores, _F32, n * beams, "scores")
    if (slots is None) != (out_slots is None):
        raise ValueError("slots and out_slots go together")
    po = [_list(t, dt, n * n_out, name) for t, dt, name in (
        (out_scores, _F32, "out_scores"), (out_tokens, _I32, "out_tokens"), (out_parents, _I32, "out_parents"))]
    pl = None if slots is None else _list(slots, _I32, n * beams, "slots")
    pol = None if slots is None else _list(out_slots, _I32, n * n_out, "out_slots")
    _here(stream, logits, scores, out_scores, out_tokens, out_parents, slots, out_slots, workspace)
    need = 0 if workspace is not None else dasc_beam_select_workspace_bytes(n, beams, vocab, n_out)
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, logits.device, stream)
    _check(LIB.dasc_beam_select(n, beams, vocab, n_out, DTYPE[logits.dtype], px, x0, x1, pc, pl, *po, pol, ws_ptr,
                                ws_bytes, _stream(stream)), "dasc_beam_select")
    del ws


def dasc_move_slots(pool, src, dst, stream=None) -> None:
    """pool[dst[g, j]] = pool[src[g, j]] as it was before the call, all moves of a group g at once.

    pool: a device tensor of slots along its first dimension, each contiguous: a state pool [n_pool,
    L, H, dk, dv], or a cache's pages.  src, dst [groups, m] or [m] int32; a move with an index outside
    the pool is left out.
    """
    if not isinstance(pool, torch.Tensor) or not pool.is_cuda:
        raise TypeError("pool must be a device tensor")
    if pool.dim() < 2 or (pool.shape[0] > 0 and not pool[0].is_contiguous()):
        raise ValueError("pool must be [n_slots, ...] with contiguous slots")
    if src.dim() == 1:
        src, dst = src[None], dst[None]
    groups, m = src.shape
    ps, s0, _ = _rows(src, _I32, (groups, m), "src")
    pd, d0, _ = _rows(dst, _I32, (groups, m), "dst")
    _here(stream, pool, src, dst)
    size = pool.element_size()
    n = pool.shape[0]
    slot = (pool.numel() // n if n else 0) * size
    _check(LIB.dasc_move_slots(pool.data_ptr(), n, slot, pool.stride(0) * size if n > 1 else slot, ps, s0, pd, d0, groups,
                               m, _stream(stream)), "dasc_move_slots")

"""Python binding of the operators in include/dasc/ops.h (argument marshalling only).

As in dasc.py: each function has the name of its C entry point and turns torch tensors into
pointers, sizes and strides; errors raise DascError.  Tensors are checked for type and device,
and that every row the kernels address lies inside them.
"""

from __future__ import annotations

import ctypes as C
import struct

import torch

from . import _lib
from ._lib import LIB
from .dasc import Shape, _check, _dev, _need, _stream

DTYPE = {torch.bfloat16: _lib.DASC_DTYPE_BF16, torch.float16: _lib.DASC_DTYPE_F16,
         torch.float32: _lib.DASC_DTYPE_F32}
ACT = {"none": _lib.DASC_ACT_NONE, "sigmoid": _lib.DASC_ACT_SIGMOID, "silu": _lib.DASC_ACT_SILU}

# The io structs are packed as bytes in one step (their ctypes classes in _lib.py give the layout)
_LINEAR_IO = struct.Struct("@6P12q")
_NORM_IO = struct.Struct("@8P11q6i2f")
assert _LINEAR_IO.size == C.sizeof(_lib.LinearIo) and _NORM_IO.size == C.sizeof(_lib.NormIo)


_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _rows(t, dtype, shape, name, dense=True):
    """(pointer, first stride, second stride) of a strided device tensor of this type and shape, of
    two or three dimensions, its last dimension contiguous if `dense`.  torch's own strides keep every
    row inside the tensor's storage.  Few attribute reads: they are most of a small call's host time."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    s = t.stride()
    if dense and s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return t.data_ptr(), s[0], s[1]


def _indices(t, n: int, name: str):
    """Pointer of n int32 indices, or None."""
    if t is None:
        return None
    p = _dev(t, _I32, name)
    if t.numel() < n:
        _need(t, n, name)
    return p


def _vector(t, dtype, n: int, name: str):
    p = _dev(t, dtype, name)
    if t.shape != (n,):
        raise ValueError(f"{name} must be [{n}], got {list(t.shape)}")
    return p


def _scratch(need: int, workspace, device, stream):
    """The caller's uint8 device tensor, or one from torch's allocator on the launch stream (as
    dasc_refresh's workspace): (tensor, pointer, bytes)."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, _dev(workspace, torch.uint8, "workspace"), workspace.numel()


def dasc_linear_attn_workspace_bytes(shape: Shape, n_req: int, n_tokens: int, max_len: int,
                                     delta: bool) -> int:
    out = C.c_size_t()
    _check(LIB.dasc_linear_attn_workspace_bytes(shape._ref, n_req, n_tokens, max_len, int(delta),
                                                C.byref(out)), "dasc_linear_attn_workspace_bytes")
    return out.value


def dasc_linear_attn(shape: Shape, layer: int, states, src_slot, dst_slot, q, k, v, g, o,
                     cu_seqlens, max_len: int, beta=None, lens=None, scale: float = 1.0,
                     workspace=None, stream=None) -> None:
    """Linear attention with a decay for each head over the tokens of every request.

    states [n_pool, L, H, dk, dv] float32; q, k [n_tokens, Hqk, dk], v and the output o
    [n_tokens, H, dv] bfloat16; log-decays g and, for the delta rule, beta [n_tokens, H]
    float32.  All but states may be strided (slices of one projection; an expanded g).
    cu_seqlens [n_req + 1] int32 gives each request's rows, max_len the longest request's
    number of tokens.  src_slot and dst_slot [n_req] int32 name the slots a request's state is
    read from (None: zero) and written to (None: not written); o None (q is then not read)
    advances the states only, by lens[i] tokens of request i if lens is given.
    """
    n_req = cu_seqlens.numel() - 1
    N, H, Hqk, dk, dv = k.shape[0], shape.n_heads, shape.n_qk_heads, shape.dk, shape.dv
    kq, hv, th = (N, Hqk, dk), (N, H, dv), (N, H)
    pk, k0, k1 = _rows(k, _BF16, kq, "k")
    pv, v0, v1 = _rows(v, _BF16, hv, "v")
    pg, g0, g1 = _rows(g, _F32, th, "g", False)
    pq = pb = po = q0 = q1 = b0 = b1 = o0 = o1 = 0
    if o is not None:
        po, o0, o1 = _rows(o, _BF16, hv, "o")
        pq, q0, q1 = _rows(q, _BF16, kq, "q")
    if beta is not None:
        pb, b0, b1 = _rows(beta, _F32, th, "beta", False)
    pc = _dev(cu_seqlens, _I32, "cu_seqlens")
    n_pool = states.shape[0]
    if states.numel() < n_pool * shape.rows * dv:
        _need(states, n_pool * shape.rows * dv, "states")
    ps = _indices(src_slot, n_req, "src_slot")
    pd = _indices(dst_slot, n_req, "dst_slot")
    pl = _indices(lens, n_req, "lens")
    need = (0 if workspace is not None else
            dasc_linear_attn_workspace_bytes(shape, n_req, N, max_len, beta is not None))
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, k.device if need else None, stream)
    io = _LINEAR_IO.pack(pq, pk, pv, pg, pb, po, q0, q1, k0, k1, v0, v1, g0, g1, b0, b1, o0, o1)
    _check(LIB.dasc_linear_attn(
        shape._ref, layer, _dev(states, _F32, "states"), n_pool, ps, pd, io, pc, pl, n_req, N, max_len,
        scale, ws_ptr, ws_bytes, _stream(stream)), "dasc_linear_attn")
    del ws


def dasc_verify_drafts_workspace_bytes(n_req: int, vocab: int) -> int:
    out = C.c_size_t()
    _check(LIB.dasc_verify_drafts_workspace_bytes(n_req, vocab, C.byref(out)),
           "dasc_verify_drafts_workspace_bytes")
    return out.value


def dasc_verify_drafts(target, draft_tokens, u_accept, u_sample, out_tokens, n_emitted, draft=None,
                       n_draft=None, workspace=None, stream=None) -> None:
    """Speculative sampling from given random numbers (see dasc/ops.h for the exact rule).

    target [n_req, max_draft + 1, vocab] and draft [n_req, max_draft, vocab] (None: drafts
    without probabilities) are probabilities in bfloat16, float16 or float32, rows contiguous;
    draft_tokens [n_req, max_draft] int32, u_accept [n_req, max_draft] and u_sample [n_req]
    float32 in [0, 1), n_draft [n_req] int32 (None: max_draft; negative: leave the request out).
    Writes out_tokens [n_req, max_draft + 1] int32 (accepted drafts, one drawn token, -1) and
    n_emitted [n_req] int32.
    """
    n_req, m, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    if target.dtype not in DTYPE:
        raise TypeError(f"target must be bfloat16, float16 or float32, got {target.dtype}")
    pt, t0, t1 = _rows(target, target.dtype, (n_req, m + 1, V), "target")
    pd, d0, d1 = None, 0, 0
    if draft is not None:
        pd, d0, d1 = _rows(draft, target.dtype, (n_req, m, V), "draft")
    pn = _indices(n_draft, n_req, "n_draft")
    px = _indices(draft_tokens, n_req * m, "draft_tokens")
    po = _indices(out_tokens, n_req * (m + 1), "out_tokens")
    pe = _indices(n_emitted, n_req, "n_emitted")
    pu = _dev(u_accept, _F32, "u_accept")
    pr = _dev(u_sample, _F32, "u_sample")
    if u_accept.numel() < n_req * m or u_sample.numel() < n_req:
        _need(u_accept, n_req * m, "u_accept")
        _need(u_sample, n_req, "u_sample")
    need = 0 if workspace is not None else dasc_verify_drafts_workspace_bytes(n_req, V)
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, target.device, stream)
    _check(LIB.dasc_verify_drafts(
        n_req, m, V, DTYPE[target.dtype], pt, t0, t1, pd, d0, d1, px, pn, pu, pr, po, pe, ws_ptr, ws_bytes,
        _stream(stream)), "dasc_verify_drafts")
    del ws


def dasc_block_norm(y, gate=None, act: str = "none", w_post=None, x=None, scale: float = 1.0,
                    channel_scale=None, w_pre=None, eps: float = 1e-6, x_out=None, h_out=None,
                    stream=None) -> None:
    """b = act(gate) * norm(y) * w_post;  x_out = x + scale * channel_scale * b;
    h_out = norm(x') * w_pre with x' before its rounding (see dasc/ops.h).

    y, gate, h_out are [rows, dim] or [outer, inner, dim] in bfloat16, float16 or float32, strided
    but for the last dimension; x and x_out have y's type or float32; w_post, w_pre and
    channel_scale [dim] have y's type or float32, all the same.  Parts left out are skipped.
    """
    if y.dtype not in DTYPE:
        raise TypeError(f"y must be bfloat16, float16 or float32, got {y.dtype}")
    if y.dim() not in (2, 3):
        raise ValueError("y must be [rows, dim] or [outer, inner, dim]")
    size, dt = tuple(y.shape), y.dtype
    deep, dim = len(size) == 3, size[-1]
    if dim == 0:
        raise ValueError("y must have columns")
    res = x if x is not None else x_out
    rdt = dt if res is None else res.dtype
    if rdt is not dt and rdt is not _F32:
        raise TypeError(f"x and x_out must be {dt} or float32, got {rdt}")
    py, y0, y1 = _rows(y, dt, size, "y")
    pg = px = pxo = ph = g0 = g1 = x0 = x1 = xo0 = xo1 = h0 = h1 = 0
    if gate is not None:
        pg, g0, g1 = _rows(gate, dt, size, "gate")
    if x is not None:
        px, x0, x1 = _rows(x, rdt, size, "x")
    if x_out is not None:
        pxo, xo0, xo1 = _rows(x_out, rdt, size, "x_out")
    if h_out is not None:
        ph, h0, h1 = _rows(h_out, dt, size, "h_out")
    weights = [t for t in (w_post, w_pre, channel_scale) if t is not None]
    wdt = weights[0].dtype if weights else dt
    if wdt is not dt and wdt is not _F32:
        raise TypeError(f"weights must be {dt} or float32, got {wdt}")
    pw = [0 if t is None else _vector(t, wdt, dim, name)
          for t, name in ((w_post, "w_post"), (w_pre, "w_pre"), (channel_scale, "channel_scale"))]
    if not deep:                           # rows have one stride
        y1 = g1 = x1 = xo1 = h1 = 0
    io = _NORM_IO.pack(py, pg, px, pxo, ph, *pw, y0, y1, g0, g1, x0, x1, xo0, xo1, h0, h1, size[0],
                       size[1] if deep else 1, dim, DTYPE[dt], DTYPE[rdt], DTYPE[wdt], ACT[act], scale,
                       eps)
    _check(LIB.dasc_block_norm(io, _stream(stream)), "dasc_block_norm")

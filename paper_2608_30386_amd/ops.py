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


def _strided(t, dtype, shape, name, dense=True):
    """Pointer of a strided device tensor of this type and shape, its last dimension contiguous
    if `dense`.  torch's own strides keep every row inside the tensor's storage."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if dense and shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return t.data_ptr()


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
    _need(states, states.shape[0] * shape.rows * dv, "states")
    bf, f32, kq, hv, th = torch.bfloat16, torch.float32, (N, Hqk, dk), (N, H, dv), (N, H)
    pk = _strided(k, bf, kq, "k")
    pv = _strided(v, bf, hv, "v")
    pg = _strided(g, f32, th, "g", False)
    pq = pb = po = None
    sq = so = (0, 0, 0)
    sb = (0, 0)
    if o is not None:
        po, so = _strided(o, bf, hv, "o"), o.stride()
        pq, sq = _strided(q, bf, kq, "q"), q.stride()
    if beta is not None:
        pb, sb = _strided(beta, f32, th, "beta", False), beta.stride()
    sk, sv, sg = k.stride(), v.stride(), g.stride()
    ps = pd = pl = None
    if src_slot is not None:
        _need(src_slot, n_req, "src_slot")
        ps = _dev(src_slot, torch.int32, "src_slot")
    if dst_slot is not None:
        _need(dst_slot, n_req, "dst_slot")
        pd = _dev(dst_slot, torch.int32, "dst_slot")
    if lens is not None:
        _need(lens, n_req, "lens")
        pl = _dev(lens, torch.int32, "lens")
    need = (0 if workspace is not None else
            dasc_linear_attn_workspace_bytes(shape, n_req, N, max_len, beta is not None))
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, states.device, stream)
    io = _LINEAR_IO.pack(pq or 0, pk, pv, pg, pb or 0, po or 0, sq[0], sq[1], sk[0], sk[1], sv[0], sv[1],
                         sg[0], sg[1], sb[0], sb[1], so[0], so[1])
    _check(LIB.dasc_linear_attn(
        shape._ref, layer, _dev(states, f32, "states"), states.shape[0], ps, pd, io,
        _dev(cu_seqlens, torch.int32, "cu_seqlens"), pl, n_req, N, max_len, scale, ws_ptr, ws_bytes,
        _stream(stream)), "dasc_linear_attn")
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
    pt, stt = _strided(target, target.dtype, (n_req, m + 1, V), "target"), target.stride()
    pd, sd = None, (0, 0)
    if draft is not None:
        pd, sd = _strided(draft, target.dtype, (n_req, m, V), "draft"), draft.stride()
    pn = None
    if n_draft is not None:
        _need(n_draft, n_req, "n_draft")
        pn = _dev(n_draft, torch.int32, "n_draft")
    _need(draft_tokens, n_req * m, "draft_tokens")
    _need(u_accept, n_req * m, "u_accept")
    _need(u_sample, n_req, "u_sample")
    _need(out_tokens, n_req * (m + 1), "out_tokens")
    _need(n_emitted, n_req, "n_emitted")
    need = 0 if workspace is not None else dasc_verify_drafts_workspace_bytes(n_req, V)
    ws, ws_ptr, ws_bytes = _scratch(need, workspace, target.device, stream)
    _check(LIB.dasc_verify_drafts(
        n_req, m, V, DTYPE[target.dtype], pt, stt[0], stt[1], pd, sd[0], sd[1],
        _dev(draft_tokens, torch.int32, "draft_tokens"), pn, _dev(u_accept, torch.float32, "u_accept"),
        _dev(u_sample, torch.float32, "u_sample"), _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(n_emitted, torch.int32, "n_emitted"), ws_ptr, ws_bytes, _stream(stream)),
        "dasc_verify_drafts")
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
    size, dt = y.shape, y.dtype
    dim = size[-1]
    res = x if x is not None else x_out
    rdt = dt if res is None else res.dtype
    if rdt is not dt and rdt is not torch.float32:
        raise TypeError(f"x and x_out must be {dt} or float32, got {rdt}")
    wdt = None
    ptrs, strides = [], []
    for t, d, name in ((y, dt, "y"), (gate, dt, "gate"), (x, rdt, "x"), (x_out, rdt, "x_out"),
                       (h_out, dt, "h_out")):
        if t is None:
            ptrs.append(0)
            strides += (0, 0)
            continue
        ptrs.append(_strided(t, d, size, name))
        s = t.stride()
        strides += (s[0], s[1] if len(s) == 3 else 0)
    for t, name in ((w_post, "w_post"), (w_pre, "w_pre"), (channel_scale, "channel_scale")):
        if t is None:
            ptrs.append(0)
            continue
        wdt = wdt or t.dtype
        if wdt is not dt and wdt is not torch.float32:
            raise TypeError(f"{name} must be {dt} or float32, got {wdt}")
        ptrs.append(_strided(t, wdt, (dim,), name))
    io = _NORM_IO.pack(*ptrs, *strides, size[0], size[1] if len(size) == 3 else 1, dim, DTYPE[dt],
                       DTYPE[rdt], DTYPE[wdt or dt], ACT[act], scale, eps)
    _check(LIB.dasc_block_norm(io, _stream(stream)), "dasc_block_norm")

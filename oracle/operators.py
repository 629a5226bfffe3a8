"""Plain fp64 definitions of the operators in include/dasc/ops.h (CPU, NumPy).

Linear attention is the recurrence itself, a token at a time; the verification of drafted
tokens works in Python integers; the norms follow their formulas.
"""

from __future__ import annotations

import numpy as np


def linear_attn(S0, q, k, v, g, beta, scale):
    """One request.  S0 [H, dk, dv], q, k [T, Hqk, dk], v [T, H, dv], g [T, H], beta [T, H] or
    None; float64.  Returns (o [T, H, dv], S_T, m) with m [H] the largest |scale| |q_t|
    |S_t[:, j]| of any token and column, the size that rounding errors of o go by."""
    S = np.array(S0, dtype=np.float64)
    H, rep = S.shape[0], S.shape[0] // k.shape[1]
    T = k.shape[0]
    o = np.zeros((T, H, S.shape[2]))
    m = np.zeros(H)
    with np.errstate(over="ignore", invalid="ignore"):
        for t in range(T):
            kt = np.repeat(k[t], rep, axis=0)
            S = S * np.exp(g[t])[:, None, None]
            u = v[t]
            if beta is not None:
                u = beta[t][:, None] * (u - np.einsum("hkv,hk->hv", S, kt))
            S = S + kt[:, :, None] * u[:, None, :]
            qt = np.repeat(q[t], rep, axis=0)
            o[t] = scale * np.einsum("hkv,hk->hv", S, qt)
            m = np.maximum(m, abs(scale) * np.linalg.norm(qt, axis=1)
                           * np.linalg.norm(S, axis=1).max(axis=1))
    return o, S, m


def whole_weight(w: float) -> int:
    """floor(min(w, 1) 2^36); 0 for negative values and NaN."""
    w = float(w)
    return int(min(w, 1.0) * 2.0 ** 36) if w > 0 else 0


def verify(target, draft, tokens, n, u_accept, u_sample):
    """One request.  target [n + 1 or more, V] and draft [n or more, V] (None: one-hot) float32
    arrays of exact values.  Returns (tokens emitted, their number)."""
    if n < 0:
        return [], 0
    V = target.shape[1]
    f32 = np.float32
    a = 0
    while a < n:
        x = int(tokens[a])
        if not 0 <= x < V:
            break
        qx = f32(draft[a][x]) if draft is not None else f32(1)
        if not f32(u_accept[a]) * qx < f32(target[a][x]):
            break
        a += 1
    p = target[a].astype(f32)
    with np.errstate(invalid="ignore"):
        if a < n and draft is not None:
            w = p - draft[a].astype(f32)
        else:
            w = p.copy()
            if a < n and 0 <= int(tokens[a]) < V:
                w[int(tokens[a])] = 0
    W = [whole_weight(x) for x in w]
    if sum(W) == 0:
        W = [whole_weight(x) for x in p]
    total, y = sum(W), -1
    if total > 0:
        u = float(u_sample)
        R = min(max(int(u * 2 ** 24), 0), 2 ** 24 - 1) if u > 0 else 0
        level = total * R >> 24
        run = 0
        for y in range(V):
            run += W[y]
            if run > level:
                break
    return [int(t) for t in tokens[:a]] + [y], a + 1


def block_norm(y, gate, act, w_post, x, scale, channel_scale, w_pre, eps):
    """float64 arrays [..., dim]; returns (x', h or None)."""
    b = np.asarray(y, dtype=np.float64)
    if w_post is not None:
        b = b / np.sqrt((b * b).mean(axis=-1, keepdims=True) + eps) * w_post
    if gate is not None:
        with np.errstate(over="ignore"):
            sig = 1.0 / (1.0 + np.exp(-gate))
        b = b * (gate * sig if act == "silu" else sig)
    b = scale * b
    if channel_scale is not None:
        b = channel_scale * b
    xp = b if x is None else x + b
    h = None
    if w_pre is not None:
        h = xp / np.sqrt((xp * xp).mean(axis=-1, keepdims=True) + eps) * w_pre
    return xp, h

"""Plain fp64 definitions of the operators in include/dasc/cache.h (CPU, NumPy).

The rotation turns complex numbers; attention is the softmax's definition over the positions that
a token sees, a token at a time; beams are a sort of all candidates; slots move through a copy.
"""

from __future__ import annotations

import numpy as np


def rotate(x, pos, inv_freq, pair_axis, adjacent):
    """x [n, heads, d], pos [n, axes] whole numbers, inv_freq [half] (fp32 values); float64 of x rotated."""
    y = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    axis = np.zeros(half, int) if pair_axis is None else np.asarray(pair_axis)
    ok = (axis >= 0) & (axis < pos.shape[1])
    # 31 bits times 24 need more than 53 (x86's long double has 64)
    p = np.where(ok, pos[:, np.where(ok, axis, 0)], 0).astype(np.longdouble)
    angle = p * np.asarray(inv_freq, dtype=np.longdouble)
    turn = (np.cos(angle).astype(np.float64) + 1j * np.sin(angle).astype(np.float64))[:, None]
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent else (slice(0, half), slice(half, 2 * half))
    z = (y[..., lo] + 1j * y[..., hi]) * turn
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def attention(q, k, v, have, n_new, kv, causal, window, scale):
    """One request.  q [n_new, Hq, d], k, v [P, Hkv, d] at the request's positions (P >= kv), have [P]
    whether a position's page exists.  Returns (o [n_new, Hq, d], lse [n_new, Hq], and for error bounds: the
    weighted mean of |v| as o, the sum of |v| over the positions seen as o, the largest scale sum |q_i k_i|
    [n_new, Hq])."""
    Hq, G = q.shape[1], q.shape[1] // k.shape[1]
    o = np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    size, total, big = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    with np.errstate(invalid="ignore", over="ignore"):
        for j in range(n_new):
            here = kv - n_new + j
            p = np.arange(kv)
            p = p[have[:kv] & ((p <= here) | (not causal)) & ((p > here - window) | (window == 0))]
            if len(p) == 0:
                continue
            for h in range(Hq):
                kk, vv = k[p, h // G], v[p, h // G]
                s = scale * (kk * q[j, h]).sum(1)
                top = s.max()
                w = np.exp(s - (top if np.isfinite(top) else 0.0))
                l = w.sum()
                if l == 0:
                    continue
                w = w / l
                o[j, h] = (w[:, None] * vv).sum(0)
                lse[j, h] = top + np.log(l)
                size[j, h] = (w[:, None] * np.abs(vv)).sum(0)
                total[j, h] = np.abs(vv).sum(0)
                big[j, h] = (scale * np.abs(kk * q[j, h]).sum(1)).max()
    return o, lse, size, total, big


def beam_select(logits, scores, n_out):
    """One request.  logits [beams, vocab], scores [beams], float64 of their exact values.  Returns lists of
    (score, token, parent), best first, -inf and -1 where candidates run out."""
    found = []
    for b in range(logits.shape[0]):
        x, start = logits[b], scores[b]
        if not np.isfinite(start) or np.isnan(x).any() or (x == np.inf).any():
            continue
        at = np.nonzero(x > -np.inf)[0]
        if len(at) == 0:
            continue
        top = x[at].max()
        lse = top + np.log(np.exp(x[at] - top).sum())
        order = at[np.lexsort((at, -x[at]))][:n_out]
        found += [(start + (x[t] - lse), b, i, int(t)) for i, t in enumerate(order)]
    found.sort(key=lambda f: (-f[0], f[1], f[2]))
    out = [(f[0], f[3], f[1]) for f in found[:n_out]]
    return out + [(-np.inf, -1, -1)] * (n_out - len(out))


def move_slots(pool, src, dst):
    """pool [n, ...]; src, dst [groups, m]."""
    old, new = pool, pool.copy()
    for s, d in zip(np.ravel(src), np.ravel(dst)):
        if 0 <= s < len(pool) and 0 <= d < len(pool):
            new[d] = old[s]
    return new

"""dasc_linear_attn's chunked form on every walk that it has, against the recurrence in 64 bits (GPU).

Which walk takes a call follows from the requests times the heads: a block holds 1, 2 or 4 (dk = 128)
column tiles of 16 that four waves share, or 4 (dk = 64) or 8 (dk = 128) tiles of a wave each, the
fewest that leave no more blocks than the chip has CUs.  The numbers of requests below, of eight heads,
lie in each of these ranges, for columns that fill the blocks and for some that do not.  Tolerances are
those of test_gpu_linear_attn.py; the oracle runs on two heads of each call.
"""

import math

import numpy as np
import pytest

import paper_2608_30386_amd as D
from oracle import operators as OO
from tests.gpu_util import announce
from tests.test_gpu_linear_attn import call, make, views

pytestmark = pytest.mark.gpu

H, HQK, HEADS = 8, 4, (0, 7)
LENGTHS = [64, 1, 130, 0, 63, 65, 17, 200, 33, 128]

# (dk, dv, requests): a walk each, from the fewest column tiles in a block to the most
WALKS = [(128, 128, 3), (128, 128, 6), (128, 128, 11), (128, 128, 20), (128, 80, 8), (128, 80, 12), (128, 80, 20),
         (128, 144, 5), (128, 144, 9), (128, 144, 12), (128, 256, 3), (128, 256, 6), (128, 256, 10),
         (64, 64, 5), (64, 64, 11), (64, 64, 20), (64, 80, 8), (64, 80, 12), (64, 144, 5), (64, 144, 9)]
FULL = [w for w in WALKS if w[1] == w[0]]


def lengths(n):
    return [LENGTHS[i % len(LENGTHS)] for i in range(n)]


def check_heads(m, src, dst, got, take=None, layer=1, scale=0.3, o_fill=7.0):
    """As check() of test_gpu_linear_attn.py, on HEADS; the other heads are held to be written whole."""
    _, Hqk, dk, dv = m["dims"]
    o, pool = got
    before = m["pool"].numpy()
    hs = list(HEADS)
    q, k, v = (x.double().numpy() for x in views(m, m["qkv"]))
    ks = [h * Hqk // H for h in hs]
    q, k, v = q[:, ks], k[:, ks], v[:, hs]
    g = m["g"].double().numpy()[:, hs]
    beta = None if m["beta"] is None else m["beta"].double().numpy()[:, hs]
    want_pool, at = before.copy(), 0
    for i, n in enumerate(m["lens"]):
        t = n if take is None else min(max(take[i], 0), n)
        s = -1 if src is None else src[i]
        S0 = before[s, layer][hs] if 0 <= s < len(before) else np.zeros((len(hs), dk, dv))
        r = slice(at, at + t)
        wo, wS, big = OO.linear_attn(S0, q[r], k[r], v[r], g[r], None if beta is None else beta[r], scale)
        tol = 2.0 ** -24 * (16 + 4 * math.sqrt(t))
        d = -1 if dst is None else dst[i]
        if 0 <= d < len(before):
            assert np.isfinite(pool[d, layer]).all()
            for j, h in enumerate(hs):
                e = np.linalg.norm(pool[d, layer, h] - wS[j])
                assert e <= tol * np.linalg.norm(wS[j]), (i, h, e / np.linalg.norm(wS[j]), tol)
            want_pool[d, layer] = pool[d, layer]
        if o is not None:
            assert np.all(o[at:at + n, :, dv:] == o_fill)
            assert np.all(o[at + t:at + n] == o_fill)
            assert np.isfinite(o[r]).all()
            err = np.abs(o[r][:, hs, :dv] - wo)
            lim = 2.0 ** -8 * 1.01 * np.abs(wo) + 2.0 ** -14 * big[None, :, None]
            assert np.all(err <= lim), (i, float((err / lim).max()))
        at += n
    np.testing.assert_array_equal(pool, want_pool)


def nan_beyond(m, take):
    """Rows that a `lens` leaves out hold NaN."""
    at = 0
    for n, t in zip(m["lens"], take):
        for name in ("qkv", "g", "beta"):
            if m[name] is not None:
                m[name][at + min(max(t, 0), n):at + n] = math.nan
        at += n


@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("dk,dv,n", WALKS)
def test_every_walk(dk, dv, n, delta):
    """With an output, and the states alone over a part of each request."""
    lens = lengths(n)
    m = make(100 + dk + dv + n, lens, H, HQK, dk, dv, delta)
    src, dst = list(range(n)), [n + (i + 1) % n for i in range(n)]
    check_heads(m, src, dst, call(m, src, dst))
    take = [max(0, x - (7, 0, 65, 1)[i % 4]) for i, x in enumerate(lens)]
    nan_beyond(m, take)
    check_heads(m, src, dst, call(m, src, dst, take=take, out=False), take)
    check_heads(m, src, None, call(m, src, None, take=take), take)


@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("dk,dv,n", FULL)
def test_strong_gates_in_place_on_every_walk(dk, dv, n, delta):
    m = make(200 + dk + n, lengths(n), H, HQK, dk, dv, delta, gates="strong")
    src = list(range(n))
    check_heads(m, src, src, call(m, src, src))


def test_windows_of_a_call_with_many_heads():
    """A delta-rule call of many heads whose chunks need more than one window of workspace, a prompt across
    each border, against two calls that meet in that prompt: the same chunks, the same bits."""
    import torch

    heads, d, cut, rest = 32, 64, 64 * 1300, 64 * 1500 + 11
    a_lens, b_lens = [100, 1, 64, 0], [30, 77, 9, 200]
    lens = [*a_lens, cut + rest, *b_lens]
    N, n = sum(lens), len(lens)
    sh = D.Shape("gdn", 1, heads, heads // 2, d, d)
    gen = torch.Generator(device="cuda").manual_seed(22)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    q = rnd(N, heads // 2, d).bfloat16()
    k = torch.nn.functional.normalize(rnd(N, heads // 2, d), dim=-1).bfloat16()
    v, g, beta = rnd(N, heads, d).bfloat16(), -rnd(N, heads).abs() * 0.05, torch.sigmoid(rnd(N, heads))
    pool = rnd(2 * n, 1, heads, d, d)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cu = lambda x: i32(np.concatenate([[0], np.cumsum(x)]))  # noqa: E731
    announce(f"linear_attn in windows: {N} tokens x {heads} heads")
    a, oa = pool.clone(), torch.zeros_like(v)
    D.dasc_linear_attn(sh, 0, a, i32(range(n)), i32(range(n, 2 * n)), q, k, v, g, oa, cu(lens), cut + rest, beta=beta)
    b, ob = pool.clone(), torch.zeros_like(v)
    at = sum(a_lens) + cut
    D.dasc_linear_attn(sh, 0, b, i32(range(5)), i32(range(n, n + 5)), q[:at], k[:at], v[:at], g[:at], ob[:at],
                       cu([*a_lens, cut]), cut, beta=beta[:at])
    D.dasc_linear_attn(sh, 0, b, i32([n + 4, *range(5, n)]), i32(range(n + 4, 2 * n)), q[at:], k[at:], v[at:], g[at:],
                       ob[at:], cu([rest, *b_lens]), rest, beta=beta[at:])
    torch.cuda.synchronize()
    assert torch.equal(oa, ob) and torch.equal(a, b)
    assert torch.isfinite(oa.float()).all() and oa[-1].abs().max() > 0


@pytest.mark.parametrize("delta", [False, True])
def test_one_workspace_for_all_batches(delta):
    """Allocated for the largest batch, used for smaller ones, which need their own parts of it; it ends
    where the query says."""
    import torch

    heads, d = 16, 64
    sh = D.Shape("gdn", 1, heads, heads, d, d)
    batches = [[2000], [1500, 700], [1000] * 4, [64, 2000, 13], [300] * 12]
    size = D.dasc_linear_attn_workspace_bytes(sh, 12, 4000, 2000, delta)
    ws = torch.empty(size + 4096, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(25)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for lens in batches:
        N, n = sum(lens), len(lens)
        q, k = (torch.nn.functional.normalize(rnd(N, heads, d), dim=-1).bfloat16() for _ in range(2))
        v, g = rnd(N, heads, d).bfloat16(), -rnd(N, heads).abs() * 0.1
        beta = torch.sigmoid(rnd(N, heads)) if delta else None
        pool, got = rnd(2 * n, 1, heads, d, d), []
        announce(f"linear_attn in a shared workspace: {lens} delta={delta}")
        for w in (None, ws[:size]):
            ws.fill_(0xA5)
            p, o = pool.clone(), torch.zeros_like(v)
            D.dasc_linear_attn(sh, 0, p, i32(range(n)), i32(range(n, 2 * n)), q, k, v, g, o,
                               i32(np.concatenate([[0], np.cumsum(lens)])), max(lens), beta=beta, workspace=w)
            got.append((p, o))
        torch.cuda.synchronize()
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert (ws[size:] == 0xA5).all()

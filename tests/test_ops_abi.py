"""The operators' C ABI: declared symbols are exported, bad arguments are refused before any launch
(CPU only: no kernel runs), and their oracle keeps the identities it stands for."""

import ctypes as C
import math
import os
import re

import numpy as np
import pytest

import paper_2608_30386_amd as D
from oracle import operators as OO
from paper_2608_30386_amd import _lib
from paper_2608_30386_amd._lib import LIB, LinearIo, NormIo, Shape

E = _lib
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000              # aligned, never dereferenced: validation fails first
ODD = 0x10002


def test_every_declared_operator_is_exported():
    text = open(os.path.join(ROOT, "include", "dasc", "ops.h")).read()
    names = re.findall(r"^int (dasc_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(_lib.EXPORTED_OPS)
    lib = C.CDLL(_lib.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def gdn(L=2, H=4, Hqk=2, dk=64, dv=64, arch=_lib.DASC_ARCH_GDN):
    return Shape(arch, L, H, Hqk, dk, dv)


def linear(shape="ok", layer=0, states=P, n_pool=2, src=P, dst=P, cu=P, lens=None, n_req=1, n_tok=4, max_len=4,
           scale=1.0, ws=P, ws_bytes=1 << 40, io_null=False, **over):
    io = LinearIo(q=P, k=P, v=P, g=P, beta=P, o=P, q_tok=128, q_head=64, k_tok=128, k_head=64, v_tok=256, v_head=64,
                  g_tok=4, g_head=1, beta_tok=4, beta_head=1, o_tok=256, o_head=64)
    for name, value in over.items():
        setattr(io, name, value)
    sh = gdn() if shape == "ok" else shape
    return LIB.dasc_linear_attn(None if sh is None else C.byref(sh), layer, states, n_pool, src, dst,
                                None if io_null else C.byref(io), cu, lens, n_req, n_tok, max_len, scale, ws, ws_bytes,
                                None)


def test_linear_attn_argument_errors():
    assert linear(None) == E.DASC_E_INVAL
    assert linear(io_null=True) == E.DASC_E_INVAL
    assert linear(gdn(dv=6)) == E.DASC_E_SHAPE
    assert linear(gdn(H=3)) == E.DASC_E_SHAPE
    for bad in (dict(layer=2), dict(layer=-1), dict(n_req=0), dict(n_tok=-1), dict(n_tok=1 << 31), dict(max_len=-1),
                dict(n_pool=0), dict(scale=math.nan), dict(scale=math.inf), dict(states=None), dict(cu=None),
                dict(states=ODD), dict(dst=None, o=None), dict(q=None), dict(k=None), dict(v=None), dict(g=None)):
        assert linear(**bad) == E.DASC_E_INVAL, bad
    for name in ("q", "k", "v", "o", "beta", "g"):
        assert linear(**{name: ODD}) == E.DASC_E_INVAL, name
    for name in ("q_tok", "q_head", "k_tok", "k_head"):
        assert linear(**{name: 68}) == E.DASC_E_INVAL, name
        assert linear(**{name: -64}) == E.DASC_E_INVAL, name
    for name in ("v_tok", "v_head", "o_tok", "o_head"):
        assert linear(**{name: 66}) == E.DASC_E_INVAL, name
    for name in ("g_tok", "g_head", "beta_tok", "beta_head"):
        assert linear(**{name: -1}) == E.DASC_E_INVAL, name
    assert linear(gdn(arch=_lib.DASC_ARCH_KDA)) == E.DASC_E_UNSUPPORTED
    assert linear(gdn(dk=48)) == E.DASC_E_UNSUPPORTED
    assert linear(gdn(dv=260)) == E.DASC_E_UNSUPPORTED


def test_linear_attn_refuses_an_output_whose_rows_overlap():
    for bad in (dict(o_tok=0), dict(o_head=0), dict(o_head=60), dict(o_tok=252), dict(o_tok=64, o_head=64),
                dict(o_tok=60, o_head=1024), dict(o_tok=64, o_head=252), dict(n_tok=1, o_head=32)):
        assert linear(**bad) == E.DASC_E_INVAL, bad


def test_linear_attn_of_no_tokens_and_no_destination():
    """A step that scores no tokens (an empty tensor's pointer is NULL) has nothing to do."""
    none = dict(q=None, k=None, v=None, g=None, beta=None)
    assert linear(n_tok=0, max_len=0, dst=None, o=None, **none) == E.DASC_OK
    assert linear(n_tok=0, max_len=0, dst=None) == E.DASC_OK
    assert linear(n_tok=0, dst=None, o=None, scale=math.nan) == E.DASC_E_INVAL


def test_linear_attn_workspace():
    out = C.c_size_t()
    ask = lambda sh, *a: LIB.dasc_linear_attn_workspace_bytes(  # noqa: E731
        None if sh is None else C.byref(sh), *a, C.byref(out))
    assert ask(None, 1, 1, 1, 0) == E.DASC_E_INVAL
    assert ask(gdn(), 0, 1, 1, 0) == E.DASC_E_INVAL
    assert ask(gdn(), 1, -1, 1, 0) == E.DASC_E_INVAL
    assert ask(gdn(), 1, 1, -1, 0) == E.DASC_E_INVAL
    assert ask(gdn(H=3), 1, 1, 1, 0) == E.DASC_E_SHAPE
    assert LIB.dasc_linear_attn_workspace_bytes(C.byref(gdn()), 1, 1, 1, 0, None) == E.DASC_E_INVAL
    for delta in (0, 1):
        assert ask(gdn(dk=128, dv=128), 3, 5000, 4000, delta) == E.DASC_OK
        if out.value:
            big = dict(n_req=3, n_tok=5000, max_len=4000)
            over = {} if delta else {"beta": None}
            assert linear(gdn(dk=128, dv=128), ws_bytes=out.value - 1, **big, **over) == E.DASC_E_WORKSPACE
            assert linear(gdn(dk=128, dv=128), ws=None, **big, **over) == E.DASC_E_WORKSPACE
            assert linear(gdn(dk=128, dv=128), ws=ODD, **big, **over) == E.DASC_E_INVAL


@pytest.mark.parametrize("delta", [0, 1])
def test_a_workspace_does_for_every_smaller_call(delta):
    out = C.c_size_t()

    def ask(sh, n, tokens, longest):
        assert LIB.dasc_linear_attn_workspace_bytes(C.byref(sh), n, tokens, longest, delta, C.byref(out)) == E.DASC_OK
        return out.value

    reqs = [1, 2, 3, 4, 5, 8, 31, 64, 300, 5000, 70000, 3000000]
    longs = [0, 1, 12, 13, 64, 800, 833, 900, 1500, 4096, 16384, 100000]
    for H, dk, dv in ((32, 128, 128), (4, 128, 256), (16, 64, 64), (1, 64, 16), (300, 128, 128), (8, 32, 64), (40000, 128, 256)):
        sh = gdn(H=H, Hqk=1, dk=dk, dv=dv, L=1)
        need = [[[ask(sh, n, min(f * longest, 2 ** 31 - 1), longest) for f in (1, 2, 7, 1000)] for longest in longs]
                for n in reqs]
        for i in range(len(reqs)):
            for j in range(len(longs)):
                for x in range(4):
                    # one step down in each: fewer requests, fewer tokens, and none so long
                    if i:
                        assert need[i - 1][j][x] <= need[i][j][x], (H, dk, dv, reqs[i], longs[j], x)
                    if j:
                        assert need[i][j - 1][x] <= need[i][j][x], (H, dk, dv, reqs[i], longs[j], x)
                    if x:
                        assert need[i][j][x - 1] <= need[i][j][x], (H, dk, dv, reqs[i], longs[j], x)
    # no tokens more, but a longer request
    sh = gdn(H=32, dk=128, dv=128)
    assert ask(sh, 4, 16384, 4096) <= ask(sh, 4, 16384, 9000)


def verify(n=1, m=2, V=100, dtype=_lib.DASC_DTYPE_F32, ws=P, ws_bytes=1 << 40, strides=(300, 100, 200, 100), **over):
    p = dict(target=P, draft=P, tokens=P, count=None, u=P, r=P, out=P, emitted=P)
    p.update(over)
    return LIB.dasc_verify_drafts(n, m, V, dtype, p["target"], strides[0], strides[1], p["draft"], strides[2],
                                  strides[3], p["tokens"], p["count"], p["u"], p["r"], p["out"], p["emitted"], ws,
                                  ws_bytes, None)


def test_verify_argument_errors():
    for bad in (dict(n=-1), dict(m=-1), dict(dtype=3), dict(dtype=-1), dict(strides=(-1, 1, 1, 1)),
                dict(strides=(1, -1, 1, 1)), dict(strides=(1, 1, -1, 1)), dict(strides=(1, 1, 1, -1)), dict(V=100000, ws=ODD)):
        assert verify(**bad) == E.DASC_E_INVAL, bad
    for bad in (dict(V=0), dict(V=(1 << 24) + 1), dict(m=1024)):
        assert verify(**bad) == E.DASC_E_SHAPE, bad
    for name in ("target", "tokens", "u", "r", "out", "emitted"):
        assert verify(**{name: None}) == E.DASC_E_INVAL, name
        assert verify(**{name: ODD}) == E.DASC_E_INVAL, name
    assert verify(draft=ODD) == E.DASC_E_INVAL and verify(count=ODD) == E.DASC_E_INVAL
    assert verify(target=P + 1, dtype=_lib.DASC_DTYPE_BF16) == E.DASC_E_INVAL
    out = C.c_size_t()
    assert LIB.dasc_verify_drafts_workspace_bytes(3, 100000, C.byref(out)) == E.DASC_OK and out.value > 0
    assert verify(n=3, V=100000, ws_bytes=out.value - 1) == E.DASC_E_WORKSPACE
    assert verify(n=3, V=100000, ws=None) == E.DASC_E_WORKSPACE
    assert verify(n=0, target=None) == E.DASC_OK
    assert LIB.dasc_verify_drafts_workspace_bytes(3, 0, C.byref(out)) == E.DASC_E_INVAL
    assert LIB.dasc_verify_drafts_workspace_bytes(-1, 5, C.byref(out)) == E.DASC_E_INVAL
    assert LIB.dasc_verify_drafts_workspace_bytes(1, 5, None) == E.DASC_E_INVAL


def norm(**over):
    io = NormIo(y=P, gate=P, x=P, x_out=P, h_out=P, w_post=P, w_pre=P, channel_scale=P, y_out=64, y_in=0, gate_out=64,
                x_row_out=64, xo_out=64, h_row_out=64, outer=3, inner=1, dim=64, dtype=_lib.DASC_DTYPE_BF16,
                res_dtype=_lib.DASC_DTYPE_F32, w_dtype=_lib.DASC_DTYPE_F32, act=_lib.DASC_ACT_SILU, scale=1.0, eps=1e-6)
    for name, value in over.items():
        setattr(io, name, value)
    return LIB.dasc_block_norm(C.byref(io), None)


def test_norm_argument_errors():
    assert LIB.dasc_block_norm(None, None) == E.DASC_E_INVAL
    for bad in (dict(y=None), dict(x_out=None, h_out=None), dict(w_pre=None), dict(dtype=9), dict(res_dtype=1),
                dict(w_dtype=1), dict(act=3), dict(act=0), dict(gate=None), dict(eps=-1.0), dict(eps=math.nan),
                dict(scale=math.inf), dict(y_out=-1), dict(gate_out=-1), dict(x_row_out=-1), dict(xo_out=0),
                dict(h_row_out=63), dict(y=P + 1), dict(gate=P + 1), dict(h_out=P + 1), dict(x=ODD), dict(x_out=ODD),
                dict(w_post=ODD), dict(w_pre=ODD), dict(channel_scale=ODD)):
        assert norm(**bad) == E.DASC_E_INVAL, bad
    for bad in (dict(outer=-1), dict(inner=0), dict(dim=0), dict(outer=1 << 20, inner=1 << 12)):
        assert norm(**bad) == E.DASC_E_SHAPE, bad
    # rows of an output may not overlap, whichever of the two strides is the longer
    assert norm(inner=2, xo_out=64, xo_in=64) == E.DASC_E_INVAL
    assert norm(inner=2, xo_out=128, xo_in=32) == E.DASC_E_INVAL
    assert norm(inner=2, xo_out=64, xo_in=128) == E.DASC_E_INVAL
    assert norm(dim=32769, y_out=40000, xo_out=40000, h_row_out=40000) == E.DASC_E_UNSUPPORTED
    assert norm(outer=0, y=None) == E.DASC_OK


def test_binding_refuses_what_the_kernels_cannot_read():
    import torch

    sh = D.Shape("gdn", 1, 2, 2, 64, 64)
    z = torch.zeros
    with pytest.raises(TypeError, match="device tensor"):
        D.dasc_linear_attn(sh, 0, z(1, 1, 2, 64, 64), None, None, z(3, 2, 64), z(3, 2, 64), z(3, 2, 64), z(3, 2),
                           z(3, 2, 64), z(2, dtype=torch.int32), 3)
    with pytest.raises(TypeError, match="device tensor"):
        D.dasc_verify_drafts(z(1, 2, 8), z(1, 1), z(1, 1), z(1), z(1, 2), z(1))
    with pytest.raises(TypeError, match="device tensor"):
        D.dasc_block_norm(z(2, 8), x_out=z(2, 8))
    with pytest.raises(TypeError, match="bfloat16, float16 or float32"):
        D.dasc_block_norm(z(2, 8, dtype=torch.float64), x_out=z(2, 8))


# ---- the oracle ---------------------------------------------------------------------------------

def test_oracle_linear_attn_identities():
    rng = np.random.default_rng(0)
    T, H, dk, dv = 9, 2, 8, 4
    q, k = rng.normal(size=(T, 1, dk)), rng.normal(size=(T, 1, dk))
    v, g = rng.normal(size=(T, H, dv)), -rng.random((T, H))
    S0 = rng.normal(size=(H, dk, dv))
    o, S, _ = OO.linear_attn(S0, q, k, v, g, None, 0.5)
    G = np.cumsum(g, 0)                                # the plain rule is a decayed sum
    for h in range(H):
        want = np.exp(G[-1, h]) * S0[h] + sum(np.exp(G[-1, h] - G[t, h]) * np.outer(k[t, 0], v[t, h]) for t in range(T))
        np.testing.assert_allclose(S[h], want, atol=1e-12)
        P = np.tril(np.exp(G[:, None, h] - G[None, :, h])) * (q[:, 0] @ k[:, 0].T)
        np.testing.assert_allclose(o[:, h], 0.5 * (P @ v[:, h] + np.exp(G[:, h])[:, None] * (q[:, 0] @ S0[h])),
                                   atol=1e-12)
    # the delta rule with unit keys and beta = 1 reads back the value it wrote
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    o, S, _ = OO.linear_attn(S0, k, k, v, g, np.ones((T, H)), 1.0)
    np.testing.assert_allclose(o, v, atol=1e-12)
    # and is the framework's recurrence
    from oracle import recurrence as OR
    beta = rng.random((T, H))
    _, S, _ = OO.linear_attn(S0, q, k, v, g, beta, 1.0)
    for h in range(H):
        np.testing.assert_allclose(S[h], OR.replay_naive(S0[h], k[:, 0], v[:, h], g[:, h], beta[:, h]),
                                   atol=1e-12)


def test_oracle_verify_draws_the_target():
    """Over many random numbers the first emitted token follows the target, whatever the draft is."""
    rng = np.random.default_rng(1)
    V, trials = 4, 20000
    p = np.array([0.5, 0.2, 0.25, 0.05], np.float32)
    q = np.array([0.1, 0.6, 0.1, 0.2], np.float32)
    count = np.zeros(V)
    for _ in range(trials):
        x = rng.choice(V, p=q.astype(np.float64) / q.sum(dtype=np.float64))
        t, _ = OO.verify(np.stack([p, p]), q[None], [x], 1, rng.random(1, dtype=np.float32), rng.random(dtype=np.float32))
        count[t[0]] += 1
    sd = np.sqrt(p * (1 - p) / trials)
    assert np.all(np.abs(count / trials - p) < 5 * sd)
    assert OO.verify(np.stack([p, p]), p[None], [2], 1, np.float32([0.999]), 0.0)[1] == 2   # p = q: kept
    assert OO.verify(np.stack([p, p]), None, [3], 1, np.float32([0.5]), 0.99)[0] == [2]     # x's weight is gone


def test_oracle_norm_identities():
    rng = np.random.default_rng(2)
    y = rng.normal(size=(3, 50))
    x, h = OO.block_norm(y, None, "none", np.ones(50), None, 1.0, None, np.ones(50), 0.0)
    np.testing.assert_allclose((x * x).mean(-1), 1, atol=1e-12)
    np.testing.assert_allclose(h, x, atol=1e-12)       # a normed row stays as it is
    x2, _ = OO.block_norm(7 * y, np.zeros((3, 50)), "sigmoid", np.ones(50), y, 2.0, None, None, 0.0)
    np.testing.assert_allclose(x2, y + x, atol=1e-12)  # scale-free, half open gate, twice

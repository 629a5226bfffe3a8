"""The paged cache's and the beams' C ABI: declared symbols are exported, bad arguments are refused before any
launch (CPU only: no kernel runs)."""

import ctypes as C
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2608_30386_amd as D
from oracle import cache as OC
from paper_2608_30386_amd import _lib
from paper_2608_30386_amd._lib import LIB, AppendIo, AttnIo, KvCache

E = _lib
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000              # aligned, never dereferenced: validation fails first
ODD = 0x10001
BIG = 1 << 31


def test_every_declared_function_is_exported():
    text = open(os.path.join(ROOT, "include", "dasc", "cache.h")).read()
    names = re.findall(r"^int (dasc_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(_lib.EXPORTED_CACHE)
    lib = C.CDLL(_lib.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and hasattr(D, n), n


def cache(**over):
    c = KvCache(k=P, v=P, k_page=2048, k_tok=128, k_head=64, v_page=2048, v_tok=128, v_head=64, n_pages=4, page_size=16,
                n_kv_heads=2, head_dim=64, dtype=E.DASC_DTYPE_BF16)
    for name, value in over.items():
        setattr(c, name, value)
    return c


def append(c="ok", null=False, **over):
    io = AppendIo(q=P, q_out=P, k=P, v=P, slots=P, pos=P, inv_freq=P, pair_axis=None, q_tok=256, q_head=64, qo_tok=256,
                  qo_head=64, k_tok=128, k_head=64, v_tok=128, v_head=64, pos_tok=1, pos_axis=1, n_tokens=3, n_q_heads=4,
                  n_axes=1, rot=64, adjacent=0)
    for name, value in over.items():
        setattr(io, name, value)
    c = cache() if c == "ok" else c
    return LIB.dasc_cache_append(None if c is None else C.byref(c), None if null else C.byref(io), None)


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=ODD), dict(dtype=E.DASC_DTYPE_F32), dict(dtype=7), dict(k_page=-2048),
              dict(v_head=-64)]
BAD_SHAPES = [dict(n_pages=0), dict(page_size=0), dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(head_dim=0),
              dict(head_dim=60), dict(head_dim=264)]


def test_append_refusals():
    assert append(None) == E.DASC_E_INVAL and append(null=True) == E.DASC_E_INVAL
    for bad in BAD_CACHES:
        assert append(cache(**bad)) == E.DASC_E_INVAL, bad
    for bad in BAD_SHAPES:
        assert append(cache(**bad)) == E.DASC_E_SHAPE, bad
    # pages, tokens or heads of the cache that overlap
    for bad in (dict(k_tok=64), dict(v_page=2000), dict(k_head=32), dict(v_tok=0), dict(k_page=0)):
        assert append(cache(**bad)) == E.DASC_E_INVAL, bad
    for bad in (dict(rot=-2), dict(rot=63), dict(rot=66), dict(n_axes=0), dict(n_axes=9), dict(n_tokens=-1),
                dict(n_tokens=BIG), dict(n_q_heads=0), dict(n_q_heads=65537)):
        assert append(**bad) == E.DASC_E_SHAPE, bad
    for bad in (dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slots=None), dict(pos=None),
                dict(inv_freq=None), dict(q=ODD), dict(q_out=ODD), dict(k=ODD), dict(v=ODD), dict(slots=P + 4),
                dict(pos=P + 2), dict(inv_freq=P + 2), dict(pair_axis=P + 2), dict(adjacent=2), dict(q_tok=-256),
                dict(q_head=-1), dict(k_tok=-1), dict(v_head=-1), dict(pos_tok=-1), dict(pos_axis=-1), dict(qo_tok=255),
                dict(qo_head=63), dict(qo_tok=0)):
        assert append(**bad) == E.DASC_E_INVAL, bad
    assert append(n_tokens=0, q=None, q_out=None, k=None, v=None, slots=None) == E.DASC_OK


def attn(c="ok", null=False, ws=P, ws_bytes=1 << 40, **over):
    io = AttnIo(q=P, o=P, lse=P, block_table=P, cu_seqlens=P, kv_lens=P, q_tok=256, q_head=64, o_tok=256, o_head=64,
                lse_tok=4, lse_head=1, table_req=8, n_tokens=3, n_req=1, n_q_heads=4, table_width=8, max_len=3, max_kv=128,
                causal=1, window=0, scale=0.1)
    for name, value in over.items():
        setattr(io, name, value)
    c = cache() if c == "ok" else c
    return LIB.dasc_cache_attn(None if c is None else C.byref(c), None if null else C.byref(io), ws, ws_bytes, None)


def test_attention_refusals():
    assert attn(None) == E.DASC_E_INVAL and attn(null=True) == E.DASC_E_INVAL
    for bad in BAD_CACHES + [dict(k=P + 8), dict(k_tok=132), dict(v_head=68)]:
        assert attn(cache(**bad)) == E.DASC_E_INVAL, bad
    for bad in BAD_SHAPES:
        assert attn(cache(**bad)) == E.DASC_E_SHAPE, bad
    for bad in (dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=65536), dict(n_tokens=-1), dict(n_tokens=BIG),
                dict(n_tokens=BIG // 2), dict(table_width=BIG // 16)):
        assert attn(**bad) == E.DASC_E_SHAPE, bad
    for bad in (dict(q=None), dict(o=None), dict(block_table=None), dict(cu_seqlens=None), dict(kv_lens=None), dict(q=P + 8),
                dict(o=P + 8), dict(lse=P + 2), dict(block_table=P + 2), dict(cu_seqlens=P + 2), dict(kv_lens=P + 2),
                dict(n_req=0), dict(table_width=-1), dict(max_len=-1), dict(max_kv=-1), dict(window=-1), dict(causal=2),
                dict(causal=-1), dict(table_req=-1), dict(scale=math.nan), dict(scale=math.inf), dict(scale=0.0),
                dict(scale=-0.1), dict(scale=1e-39), dict(scale=3e38), dict(q_tok=-256), dict(q_tok=252), dict(q_head=68),
                dict(o_tok=252), dict(o_tok=0), dict(o_head=56), dict(o_tok=64), dict(lse_tok=0), dict(lse_tok=3),
                dict(lse_head=0)):
        assert attn(**bad) == E.DASC_E_INVAL, bad
    assert attn(n_tokens=0, q=None, o=None) == E.DASC_OK


def attn_bytes(*sizes):
    out = C.c_size_t()
    assert LIB.dasc_cache_attn_workspace_bytes(*sizes, C.byref(out)) == E.DASC_OK
    return out.value


def test_attention_workspace():
    out = C.c_size_t()
    ask = lambda *a: LIB.dasc_cache_attn_workspace_bytes(*a, C.byref(out))  # noqa: E731
    assert LIB.dasc_cache_attn_workspace_bytes(1, 1, 4, 2, 64, 1, 1, None) == E.DASC_E_INVAL
    assert ask(0, 1, 4, 2, 64, 1, 1) == E.DASC_E_INVAL
    assert ask(1, 1, 4, 2, 64, -1, 1) == E.DASC_E_INVAL and ask(1, 1, 4, 2, 64, 1, -1) == E.DASC_E_INVAL
    for bad in ((1, -1, 4, 2, 64, 1, 1), (1, 1, 4, 3, 64, 1, 1), (1, 1, 4, 0, 64, 1, 1), (1, 1, 4, 2, 65, 1, 1)):
        assert ask(*bad) == E.DASC_E_SHAPE, bad
    need = attn_bytes(1, 1, 4, 2, 64, 1, 128 * 16)
    assert need > 0
    big = dict(n_tokens=1, max_len=1, max_kv=128 * 16, table_width=128)
    assert attn(ws=None, **big) == E.DASC_E_WORKSPACE
    assert attn(ws_bytes=16, **big) == E.DASC_E_WORKSPACE
    assert attn(ws=P + 8, **big) == E.DASC_E_INVAL


def test_an_attention_workspace_does_for_every_smaller_call():
    rng = np.random.default_rng(0)
    for _ in range(300):
        hkv = int(rng.choice([1, 2, 8, 16]))
        hq, d = hkv * int(rng.choice([1, 2, 5, 8, 16])), int(rng.choice([8, 64, 96, 128, 256]))
        n_req, most, kv = int(rng.integers(1, 300)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 16))
        tokens = int(rng.integers(0, n_req * most + 1))
        small = (int(rng.integers(1, n_req + 1)), int(rng.integers(0, tokens + 1)), hq, hkv, d,
                 int(rng.integers(0, most + 1)), int(rng.integers(0, kv + 1)))
        assert attn_bytes(*small) <= attn_bytes(n_req, tokens, hq, hkv, d, most, kv), small


def select(n_req=2, beams=3, vocab=100, n_out=4, dtype=2, logits=P, x0=300, x1=100, scores=P, slots=P, out=(P, P, P, P), ws=P,
           ws_bytes=1 << 40):
    return LIB.dasc_beam_select(n_req, beams, vocab, n_out, dtype, logits, x0, x1, scores, slots, *out, ws, ws_bytes, None)


def test_beam_select_refusals():
    for bad in (dict(n_req=-1), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(n_out=0),
                dict(n_out=65), dict(n_req=1 << 20, beams=17)):
        assert select(**bad) == E.DASC_E_SHAPE, bad
    for bad in (dict(dtype=3), dict(logits=None), dict(scores=None), dict(out=(None, P, P, P)), dict(out=(P, None, P, P)),
                dict(out=(P, P, None, P)), dict(out=(P, P, P, None)), dict(slots=None), dict(logits=P + 2),
                dict(logits=ODD, dtype=0), dict(x0=-1), dict(x1=-1), dict(scores=P + 2), dict(slots=P + 2),
                dict(out=(P + 2, P, P, P)), dict(out=(P, P, P, P + 1)), dict(ws=P + 8)):
        assert select(**bad) == E.DASC_E_INVAL, bad
    assert select(n_req=0, logits=None) == E.DASC_OK
    out = C.c_size_t()
    assert LIB.dasc_beam_select_workspace_bytes(2, 3, 100, 4, C.byref(out)) == E.DASC_OK
    assert select(ws_bytes=out.value - 1) == E.DASC_E_WORKSPACE and select(ws=None) == E.DASC_E_WORKSPACE
    assert LIB.dasc_beam_select_workspace_bytes(2, 3, 100, 4, None) == E.DASC_E_INVAL
    assert LIB.dasc_beam_select_workspace_bytes(2, 0, 100, 4, C.byref(out)) == E.DASC_E_SHAPE


def move(pool=P, n=4, size=64, stride=64, src=P, s0=2, dst=P, d0=2, groups=1, m=2):
    return LIB.dasc_move_slots(pool, n, size, stride, src, s0, dst, d0, groups, m, None)


def test_move_slots_refusals():
    for bad in (dict(groups=-1), dict(groups=65536), dict(m=-1), dict(m=65)):
        assert move(**bad) == E.DASC_E_SHAPE, bad
    for bad in (dict(pool=None), dict(src=None), dict(dst=None), dict(pool=P + 8), dict(src=P + 2), dict(dst=P + 2), dict(n=0),
                dict(size=0), dict(size=24), dict(stride=72), dict(stride=48), dict(s0=-1), dict(d0=-1)):
        assert move(**bad) == E.DASC_E_INVAL, bad
    assert move(groups=0, pool=None) == E.DASC_OK and move(m=0, src=None) == E.DASC_OK


def test_the_binding_takes_device_tensors_only():
    x = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        D.dasc_cache_append(x, x, i.long(), x[0, :4], x[0, :4])
    with pytest.raises(TypeError):
        D.dasc_cache_attn(x, x, i[None], i[:1], x[0], x[0], i[:2], 1)
    with pytest.raises(TypeError):
        D.dasc_beam_select(torch.zeros(1, 2, 9), torch.zeros(1, 2), *(torch.zeros(1, 2) for _ in range(3)))
    with pytest.raises(TypeError):
        D.dasc_move_slots(x, i, i)


def test_the_oracle_keeps_its_identities():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 8))
    inv = np.array([1.0, 0.5, 0.1])
    for adjacent in (False, True):
        at0 = OC.rotate(x, np.zeros((3, 1), int), inv, None, adjacent)
        np.testing.assert_array_equal(at0, x)
        y = OC.rotate(x, np.array([[3], [4], [5]]), inv, None, adjacent)
        back = OC.rotate(y, -np.array([[3], [4], [5]]), inv, None, adjacent)
        np.testing.assert_allclose(back, x, atol=1e-14)
        # products depend on the distance alone
        a, b = x[:1], x[1:2]
        dot = lambda s: (OC.rotate(a, np.array([[s]]), inv, None, adjacent)  # noqa: E731
                         * OC.rotate(b, np.array([[s + 9]]), inv, None, adjacent)).sum()
        assert abs(dot(0) - dot(1000)) < 1e-12
    q, k, v = rng.standard_normal((2, 2, 4)), rng.standard_normal((5, 1, 4)), rng.standard_normal((5, 1, 4))
    o, lse, *_ = OC.attention(q, k, v, np.ones(5, bool), 2, 5, True, 1, 0.5)
    np.testing.assert_allclose(o[1], np.repeat(v[4], 2, 0))                 # a window of one: the token itself
    np.testing.assert_allclose(lse[1], 0.5 * (q[1] * k[4]).sum(-1))
    o, *_ = OC.attention(q * 0, k, v, np.ones(5, bool), 2, 5, True, 0, 0.5)
    np.testing.assert_allclose(o[0], np.repeat(v[:4].mean(0), 2, 0))
    z = rng.standard_normal((2, 6))
    got = OC.beam_select(z, np.array([0.0, -1.0]), 12)
    flat = (z - np.log(np.exp(z).sum(1, keepdims=True)) + np.array([[0.0], [-1.0]])).ravel()
    np.testing.assert_allclose([g[0] for g in got], np.sort(flat)[::-1])
    assert [g[2] * 6 + g[1] for g in got] == np.argsort(-flat).tolist()


def test_strides_of_dimensions_of_one_element_do_not_matter():
    one = dict(n_pages=1, k_page=3, v_page=1 << 40)
    flat = dict(page_size=1, k_tok=5, v_tok=1 << 30, k_page=128, v_page=128)
    single = dict(n_kv_heads=1, k_head=3, v_head=9)
    none = dict(n_tokens=0, q=None, k=None, v=None, slots=None)
    for c in (one, flat, single):
        assert append(cache(**c), q_out=None, **none) == E.DASC_OK, c
        assert attn(cache(**c), n_tokens=0, q=None, o=None) == E.DASC_OK, c
    # a call that lacks nothing but its workspace
    big = dict(ws=None, n_tokens=1, max_len=1, max_kv=128 * 16, table_width=128)
    for odd in (dict(q_tok=257, o_tok=3, lse_tok=0), dict(q_tok=0, o_tok=0)):
        assert attn(**big, **odd) == E.DASC_E_WORKSPACE, odd
    assert attn(cache(**single), n_q_heads=1, q_head=3, o_head=1, lse_head=0, **big) == E.DASC_E_WORKSPACE
    assert attn(cache(**one), **big) == E.DASC_E_WORKSPACE


def test_rows_that_end_where_the_next_ones_start():
    """Three heads 80 elements apart, of 64: 224 elements a token, not 240.  The last row counts with its width alone."""
    none = dict(n_tokens=0, q=None, k=None, v=None, slots=None)
    close = dict(n_kv_heads=3, k_head=80, v_head=80, k_tok=224, v_tok=224, k_page=15 * 224 + 224, v_page=3584)
    assert append(cache(**close), q_out=None, **none) == E.DASC_OK
    for bad in (dict(k_tok=223), dict(v_page=3583), dict(v_head=63)):
        assert append(cache(**{**close, **bad}), q_out=None, **none) == E.DASC_E_INVAL, bad
    big = dict(ws=None, max_len=1, max_kv=128 * 16, table_width=128, n_q_heads=2)
    for o_tok, o_head, want in ((144, 80, E.DASC_E_WORKSPACE), (136, 80, E.DASC_E_INVAL), (64, 192, E.DASC_E_WORKSPACE),
                                (64, 184, E.DASC_E_INVAL), (72, 208, E.DASC_E_WORKSPACE)):
        assert attn(o_tok=o_tok, o_head=o_head, lse=None, **big) == want, (o_tok, o_head)

"""Attention over the paged cache where it can go wrong by its schedule or its number range (GPU).

Tolerances are those of tests/test_gpu_cache_attn.py; what is not finite has to be equal, infinities with their sign.

Weights in fp16: the operand is 2^(s - m + 7) with the base m at most 8 below the row's maximum, off by at most 2^-25
where it is subnormal, so by 2^-32 of the largest weight: 2^-32 sum |v| in the output, and 2^-25 where that is
subnormal itself.
"""

import numpy as np
import pytest

from oracle import cache as OC
from tests.gpu_util import announce
from tests.test_gpu_cache_attn import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,page", [(136, 16), (160, 7), (256, 16), (256, 100)])
def test_waves_of_a_tile_that_leave_steps_out(d, page, dtype):
    """Heads above 128, tiles of many rows: with a window the tile's first steps are seen by its first wave alone, so the
    others pass them without products and are the first to store the next keys.  Every call gives the same bits, those
    of the formula."""
    import torch

    announce(f"cache attn: waves apart, d={d} pages of {page} {dtype}")
    c = make([(129, 700), (260, 300), (70, 70)], dtype=dtype, hq=4, hkv=2, d=d, page=page, seed=11)
    for window in (0, 1, 40, 90):
        o, s = call(c, window=window)
        check(c, o, s, window=window)
        for _ in range(10):
            o2, s2 = call(c, window=window)
            assert torch.equal(o, o2) and torch.equal(s, s2)


def want(c, i, causal=True, window=0):
    """The oracle's results of request i (o, lse, weighted mean and sum of |v|, largest scale sum |q k|) and its rows."""
    import torch

    n, kv, n_pages = c["reqs"][i][0], int(c["kv"][i]), c["kc"].shape[0]
    rows = slice(int(c["cu"][i]), int(c["cu"][i]) + n)
    p = np.arange(kv)
    pages = c["table"][i, p // c["page"]]
    have = (pages >= 0) & (pages < n_pages)
    at = torch.tensor(np.where(have, pages, 0), device="cuda"), torch.tensor(p % c["page"], device="cuda")
    k, v = (x[at].double().cpu().numpy() for x in (c["kc"], c["vc"]))
    q = c["q"][rows].double().cpu().numpy()
    return OC.attention(q, k, v, have, n, kv, causal, window, q.shape[2] ** -0.5), rows


def strict(c, **how):
    """check(), and equal values where the result is not finite."""
    o, s = call(c, **how)
    mask = {k: v for k, v in how.items() if k in ("causal", "window")}
    check(c, o, s, **mask)
    for i in range(len(c["reqs"])):
        (wo, wl, *_), rows = want(c, i, **mask)
        for got, exact in ((o[rows], wo), (s[rows], wl)):
            got = got.double().cpu().numpy()
            odd = ~np.isfinite(exact)
            np.testing.assert_array_equal(got[odd], exact[odd])
            assert np.isfinite(got[~odd]).all()


@pytest.mark.parametrize("stale", [float("nan"), float("inf")])
@pytest.mark.parametrize("page", [7, 16])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 8, 1), (256, 4, 2)])
def test_values_that_are_not_finite_reach_those_that_see_them(d, hq, hkv, dtype, page, stale):
    announce(f"cache attn: values not finite, d={d} pages of {page} {dtype} {stale}")
    for reqs in ([(1, 37), (1, 200), (1, 1)], [(6, 90), (4, 33)], [(12, 90), (20, 61)], [(70, 150), (129, 129)]):
        c = make(reqs, dtype=dtype, hq=hq, hkv=hkv, d=d, page=page, stale=stale, seed=6)
        strict(c)
        c["table"][0, 1] = -1                   # a hole
        if c["table"].shape[1] > 3:
            c["table"][-1, 2] = c["kc"].shape[0]
        for i, (n, kv) in enumerate(reqs):      # among the new tokens, of one sign and of both in a column
            for back, column, value in ((n // 3, d // 2, stale), (n // 2, 3, -stale), (0, d // 2, -stale), (n - 1, 5, stale)):
                p = kv - 1 - back
                at = c["table"][i, p // page]
                if 0 <= at < c["kc"].shape[0]:
                    c["vc"][at, p % page, hkv - 1, column] = value
        strict(c)
        strict(c, window=7)
        strict(c, causal=False)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 7), (256, 16)])
@pytest.mark.parametrize("reqs", [[(1, 40), (1, 6000)], [(5, 300)], [(20, 61), (11, 3000)], [(70, 150)], [(100, 4100)]],
                         ids=lambda r: "-".join(f"{n}of{kv}" for n, kv in r))
def test_scores_that_are_not_finite(reqs, d, page, dtype):
    """A score of +inf: its row's log-sum is +inf and its output, inf / inf, NaN; of NaN: both NaN; of -inf: no weight."""
    announce(f"cache attn: scores not finite {reqs} d={d} {dtype}")
    for seed, value in enumerate((float("inf"), -float("inf"), float("nan"))):
        c = make(reqs, dtype=dtype, hq=4, hkv=2, d=d, page=page, seed=20 + seed)
        for i, (n, kv) in enumerate(reqs):
            for p in (kv - 1 - n // 2, kv // 3):
                c["kc"][c["table"][i, p // page], p % page, 0, 5] = value
        c["q"][0, 1, :] = 0.0                   # 0 times an infinity is NaN
        strict(c)
        strict(c, window=9)
    c = make(reqs, dtype=dtype, hq=4, hkv=2, d=d, page=page, seed=30)
    c["q"][0, 0, 3] = float("inf")              # scores of both infinities
    c["q"][-1, 3, 0] = float("nan")
    strict(c)


@pytest.mark.parametrize("sink", [0, 9001])
@pytest.mark.parametrize("n,d", [(1, 64), (9, 128), (20, 64), (70, 128), (40, 256)])
def test_many_small_weights_beside_a_large_one(n, d, sink):
    """30011 positions, one with 2^25.4 times the others' weight and a value of 0: in fp16 the others are
    subnormal beside it, and all of the output."""
    import torch

    announce(f"cache attn: small weights, {n} tokens d={d} sink at {sink}")
    kv, page = 30011, 16
    c = make([(n, kv)], dtype="float16", hq=2, hkv=1, d=d, page=page, seed=40)
    c["kc"][:] = 0
    c["q"][:] = 0
    c["q"][..., 1] = 8.0
    at = (c["table"][0, sink // page], sink % page, 0)
    c["kc"][at + (1,)] = 25.4 * np.log(2) * d ** 0.5 / 8
    c["vc"][:] = 0.5 + torch.rand(c["vc"].shape, device="cuda", generator=torch.Generator("cuda").manual_seed(41)).half()
    c["vc"][at] = 0
    for over in ({}, dict(max_kv=10)):          # cut into pieces, and whole
        o, s = call(c, **over)
        (wo, wl, size, total, big), _ = want(c, 0)
        ds = 2.0 ** -24 * (d + 8) * big + 2.0 ** -22
        tol = (2.0 ** -11 * (np.abs(wo) + size) + 2 * (ds[..., None] + kv * 2.0 ** -24) * size + 2.0 ** -32 * total
               + 2.0 ** -25)
        err = np.abs(o.double().cpu().numpy() - wo)
        assert (err <= tol).all(), (over, (err / tol).max())
        assert (np.abs(s.double().cpu().numpy() - wl) <= ds + kv * 2.0 ** -24 + 2.0 ** -22 * (np.abs(wl) + 1)).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d", [(1, 64), (9, 128), (70, 128), (40, 256)])
def test_far_scores(n, d, dtype):
    """Scores of 2^26 to 2^27, whose fp32 neighbours are 4 to 8 apart: their rounding decides which positions weigh
    something, but weights stay numbers of the type and their mean stays among the values, up to a rounding of the
    weights and one of the output."""
    import torch

    announce(f"cache attn: far scores, {n} tokens d={d} {dtype}")
    c = make([(n, 900)], dtype=dtype, hq=2, hkv=1, d=d, seed=50)
    g = torch.Generator("cuda").manual_seed(51)
    for x in (c["q"], c["kc"]):
        x.copy_((torch.rand(x.shape, device="cuda", generator=g) * 100 + 3e3).to(c["dt"]))
    for sign in (1, -1):
        c["q"].mul_(sign)
        for over in ({}, dict(max_kv=10)):
            o, s = call(c, **over)
            assert torch.isfinite(s).all() and torch.isfinite(o).all()
            assert float(o.float().abs().max()) <= float(c["vc"].float().abs().max()) * (1 + torch.finfo(c["dt"]).eps)
            exact = c["q"].double() @ c["kc"].double().flatten(0, -2).T * d ** -0.5
            assert ((s.double() - sign * exact.abs().mean()).abs() <= 0.02 * exact.abs().mean()).all()


def test_strides_of_dimensions_of_one_element():
    """They are never used, so any will do: a token of a row that is no multiple of 8 elements wide, a cache of one page,
    of pages of one token, of one head."""
    import torch

    announce("cache attn: strides of single elements")
    c = make([(1, 9)], hq=4, hkv=2, d=64, page=16)
    c["kc"], c["vc"] = (x[:1].as_strided((1, 16, 2, 64), (77777, 128, 64, 1)) for x in (c["kc"], c["vc"]))
    c["table"][:] = 0
    c["q"] = c["q"].as_strided((1, 4, 64), (259, 64, 1))
    o, s = call(c, o=torch.zeros(300, dtype=c["dt"], device="cuda").as_strided((1, 4, 64), (13, 64, 1)))
    check(c, o, s)
    c = make([(3, 70)], hq=4, hkv=1, d=64, page=1)
    c["kc"], c["vc"] = (x.as_strided(x.shape, (64, 3, 5, 1)) for x in (c["kc"], c["vc"]))
    o, s = call(c)
    check(c, o, s)
    c = make([(5, 20)], hq=1, hkv=1, d=64)
    c["q"] = c["q"].as_strided((5, 1, 64), (64, 1, 1))
    o, s = call(c)
    check(c, o, s)


@pytest.mark.parametrize("n", [3, 70])
def test_rows_that_end_where_the_next_ones_start(n):
    """Two heads 80 elements apart of 64, tokens 144: the 16 elements between the heads stay as they were."""
    import torch

    announce(f"cache attn: close rows, {n} tokens")
    c = make([(n, n + 50)], hq=2, hkv=1, d=64)
    flat = torch.full((n * 144,), 5.0, dtype=c["dt"], device="cuda")
    o, s = call(c, o=flat.as_strided((n, 2, 64), (144, 80, 1)))
    check(c, o, s)
    assert (flat.as_strided((n, 16), (144, 1), 64) == 5.0).all()

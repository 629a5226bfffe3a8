"""dasc_linear_attn where its inputs are not finite, or its decays grow: what a token may not reach (GPU).

The chunked form multiplies whole blocks of a triangular matrix, zeros among them, and zero times an
infinity is NaN: a token's NaN or infinity must still not reach the tokens before it, other columns or
other requests.  Here the chunked form is held to the token-by-token form (max_len of 0 chooses it), which
computes a token's row from the state and that token alone: the same places are infinite or NaN, and
what is finite agrees within the tolerances of test_gpu_linear_attn.py, taken twice, once for each form.
Every walk of the chunked form is taken (see test_gpu_linear_tiles.py).
"""

import math

import numpy as np
import pytest

from tests.test_gpu_linear_attn import call, check, make, views
from tests.test_gpu_linear_tiles import FULL, H, HQK, WALKS, lengths

pytestmark = pytest.mark.gpu


def same(m, got, want, scale=0.3):
    (o, pool), (wo, wpool) = got, want
    with np.errstate(invalid="ignore", over="ignore"):
        for a, b in ((o, wo), (pool, wpool)):
            if a is not None:
                np.testing.assert_array_equal(np.isnan(a), np.isnan(b))
                np.testing.assert_array_equal(np.where(np.isinf(a), a, 0), np.where(np.isinf(b), b, 0))
        fin = np.isfinite(wpool)
        x, y = np.where(fin, pool, 0).astype(np.float64), np.where(fin, wpool, 0).astype(np.float64)
        T = max(m["lens"])
        tol = 2 * 2.0 ** -24 * (16 + 4 * math.sqrt(T))
        err, size = np.linalg.norm(x - y, axis=(-2, -1)), np.linalg.norm(y, axis=(-2, -1))
        assert np.all(err <= tol * size), float((err / np.maximum(size, 1e-30)).max())
        if o is not None:
            fin = np.isfinite(wo)
            x, y = np.where(fin, o, 0).astype(np.float64), np.where(fin, wo, 0).astype(np.float64)
            lim = 2 * 2.0 ** -8 * 1.01 * np.abs(y) + 2 * 2.0 ** -14 * largest(m, scale)
            assert np.all(np.abs(x - y) <= lim), float((np.abs(x - y) / np.maximum(lim, 1e-30)).max())


def largest(m, scale):
    """|scale| |q| times a bound on the columns of the states: |S_0| and |v| of all tokens before."""
    q, _, v = (np.nan_to_num(x.double().numpy(), nan=0, posinf=0, neginf=0) for x in views(m, m["qkv"]))
    S0 = np.nan_to_num(m["pool"].numpy(), nan=0, posinf=0, neginf=0)
    return scale * np.linalg.norm(q, axis=-1).max() * (np.linalg.norm(S0, axis=-2).max() + np.abs(v).max() * 8)


def plant(m, what, value, rows):
    """`value` at one element of the tokens `rows` of a tensor, or of requests' first states."""
    Hh, Hqk, dk, dv = m["dims"]
    q, k, v = views(m, m["qkv"])
    for j, r in enumerate(rows):
        if what == "v":
            v[r, (3 * j) % Hh, (5 * j + 17) % dv] = value
        elif what == "k":
            k[r, j % Hqk, (7 * j + 3) % dk] = value
        elif what == "q":
            q[r, j % Hqk, (7 * j + 3) % dk] = value
        elif what == "state":
            m["pool"][j % len(m["lens"]), 1, (3 * j) % Hh, (5 * j) % dk, (11 * j + 1) % dv] = value
        elif m[what] is not None:
            m[what][r, (3 * j) % Hh] = value


def both(m, src, dst, **kw):
    return call(m, src, dst, **kw), call(m, src, dst, max_len=0, **kw)


def marked(lens):
    """A token in the middle of most requests, at a chunk's start, its end and between."""
    at = np.cumsum([0] + lens[:-1])
    return [int(a + (0, 63, 40, 17, n - 1)[i % 5] % n) for i, (a, n) in enumerate(zip(at, lens)) if n > 0 and i % 4 != 3]


@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("dk,dv,n", WALKS)
def test_what_is_not_finite_stays_behind_its_token(dk, dv, n, delta):
    lens = lengths(n)
    src, dst = list(range(n)), [n + (i + 1) % n for i in range(n)]
    for what, value in (("v", math.inf), ("v", math.nan), ("k", math.nan), ("state", math.inf)):
        m = make(300 + dk + dv + n, lens, H, HQK, dk, dv, delta)
        plant(m, what, value, marked(lens))
        same(m, *both(m, src, dst))
        if what == "v":
            same(m, *both(m, src, src, out=False))
            same(m, *both(m, src, src))


@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("what,value", [("k", math.inf), ("beta", math.nan), ("beta", math.inf), ("g", math.nan),
                                        ("state", math.nan), ("v", -math.inf)])
def test_other_places_that_are_not_finite(what, value, delta):
    for dk, dv, n in ((128, 128, 3), (128, 128, 20), (64, 64, 5)):
        lens = lengths(n)
        m = make(310 + n, lens, H, HQK, dk, dv, delta)
        plant(m, what, value, marked(lens))
        src = list(range(n))
        same(m, *both(m, src, src))


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("dk,dv,n", FULL)
def test_a_query_reaches_its_own_outputs_only(dk, dv, n, delta, value):
    """An infinite query's own row is infinite or NaN; every other row keeps its bits."""
    lens = lengths(n)
    src, dst = list(range(n)), [n + (i + 1) % n for i in range(n)]
    m = make(320 + dk + n, lens, H, HQK, dk, dv, delta)
    o0, pool0 = call(m, src, dst)
    rows = marked(lens)
    plant(m, "q", value, rows)
    o1, pool1 = call(m, src, dst)
    np.testing.assert_array_equal(pool0, pool1)
    hit = np.zeros(o0.shape[:2], bool)
    for j, r in enumerate(rows):
        hit[r, [h for h in range(H) if h * HQK // H == j % HQK]] = True
    np.testing.assert_array_equal(o0[~hit], o1[~hit])
    assert not np.isfinite(o1[hit][:, :dv]).any()


@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("lens,hint", [([1500, 700], None), ([2500, 1, 0, 70], None), ([40, 2900], 1300)])
def test_segments_of_the_plain_rule(lens, hint, out):
    """Requests split over their length: an infinity in one segment reaches those behind it alone."""
    for dk in (64, 128):
        m = make(330 + dk, lens, 2, 1, dk, dk, False)
        src = list(range(len(lens)))
        plant(m, "v", math.inf, [3, 901, lens[0] - 1, sum(lens) - 5])
        same(m, call(m, src, src, max_len=hint, out=out), call(m, src, src, max_len=0, out=out))


def test_windows():
    """A delta-rule call in more than one window, a NaN in the request that crosses the border."""
    import torch

    import paper_2608_30386_amd as D
    from tests.gpu_util import announce

    Hh, d, N = 8, 64, 64 * 4400 + 3
    sh = D.Shape("gdn", 1, Hh, Hh // 2, d, d)
    gen = torch.Generator(device="cuda").manual_seed(23)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    q, k = rnd(N, Hh // 2, d).bfloat16(), torch.nn.functional.normalize(rnd(N, Hh // 2, d), dim=-1).bfloat16()
    v, g, beta = rnd(N, Hh, d).bfloat16(), -rnd(N, Hh).abs() * 0.05, torch.sigmoid(rnd(N, Hh))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cu = i32(0, 100, N)
    outs = []
    bad = N - 3000
    for planted in (False, True):
        if planted:
            v[bad, 5, 9] = math.nan
        pool, o = torch.ones(2, 1, Hh, d, d, device="cuda"), torch.zeros_like(v)
        announce(f"linear_attn in windows, planted={planted}")
        D.dasc_linear_attn(sh, 0, pool, i32(0, 1), i32(0, 1), q, k, v, g, o, cu, N - 100, beta=beta)
        outs.append((pool, o))
    torch.cuda.synchronize()
    (p0, o0), (p1, o1) = outs
    hit = torch.zeros(Hh, d, dtype=torch.bool, device="cuda")
    hit[5, 9] = True
    assert torch.isnan(o1[bad:, 5, 9].float()).all() and torch.isnan(p1[1, 0, 5, :, 9]).all()
    # the column's tile was walked by token: finite, and the same but for rounding
    assert torch.isfinite(o1[:bad].float()).all() and torch.isfinite(o1[bad:][:, ~hit].float()).all()
    e = (o1[:bad].float() - o0[:bad].float()).abs().max()
    assert e <= 2 ** -6 * o0.abs().max(), e
    assert torch.equal(p0[0], p1[0])
    fin = torch.isfinite(p1[1, 0])
    assert (~fin).sum() == d and (p1[1, 0][fin] - p0[1, 0][fin]).abs().max() < 1e-4 * p0[1].abs().max()


@pytest.mark.parametrize("delta", [False, True])
@pytest.mark.parametrize("dk,dv,n", FULL)
def test_growth_over_a_state_of_zero(dk, dv, n, delta):
    """Log-decays that sum to more than fp32's exponential holds, over a state that is zero until late."""
    lens = [max(1, x) for x in lengths(n)]
    m = make(340 + dk + n, lens, H, HQK, dk, dv, delta)
    at = 0
    for x in lens:
        m["g"][at:at + x] = 1.5
        late = at + max(0, x - 9)
        m["qkv"][at:late, 2 * HQK * dk:2 * HQK * dk + H * dv] = 0
        at += x
    dst = list(range(n))
    got = call(m, None, dst)
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all()
    same(m, got, call(m, None, dst, max_len=0))
    if n < 12:
        check(m, None, dst, got)


def test_growth_over_a_segment():
    """A decay over a segment that fp32 does not hold, over a state of zero: 60 chunks of 64 heads go in
    segments of 15, each of a growth of e^96."""
    heads, n = 64, 3840
    m = make(350, [n], heads, heads, 64, 64, False)
    m["g"][:] = 0.1
    m["g"][n - 50:] = -0.01
    m["qkv"][:n - 50, 2 * heads * 64:] = 0
    for out in (True, False):
        got = call(m, None, [1], out=out)
        assert np.isfinite(got[1]).all() and (not out or np.isfinite(got[0]).all())
        same(m, got, call(m, None, [1], max_len=0, out=out))


@pytest.mark.parametrize("delta", [False, True])
def test_a_scale_near_the_largest_number(delta):
    """Times a factor that grows a little it would pass fp32; over values of zero the outputs are zero."""
    m = make(351, [100, 30], 2, 1, 64, 64, delta)
    m["g"][:] = 0.1
    m["qkv"][:, 2 * 64:2 * 64 + 2 * 64] = 0
    check(m, None, [0, 1], call(m, None, [0, 1], scale=3e38), scale=3e38)


def test_growth_after_a_reset():
    """A segment of 127 chunks that begins with a reset and then grows, over values of zero, by as much as
    the kernels let a reset shrink: the reset holds."""
    import torch

    import paper_2608_30386_amd as D
    from tests.gpu_util import announce

    heads, d, n = 64, 64, 4 * 127 * 64
    gen = torch.Generator(device="cuda").manual_seed(24)
    q, k = (torch.randn((n, 1, d), device="cuda", generator=gen).bfloat16() for _ in range(2))
    v, o = torch.zeros((2, n, heads, d), dtype=torch.bfloat16, device="cuda")
    g = torch.full((n, heads), 0.17, device="cuda")
    g[0], g[127 * 64:] = -math.inf, 0.0
    pool = torch.randn((2, 1, heads, d, d), device="cuda", generator=gen)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    announce(f"linear_attn: {n} tokens that grow after a reset")
    for out in (o, None):
        pool[1] = 3.0
        D.dasc_linear_attn(D.Shape("gdn", 1, heads, 1, d, d), 0, pool, i32(0), i32(1), q, k, v, g, out, i32(0, n), n)
        torch.cuda.synchronize()
        assert not pool[1].any() and not o.any()


@pytest.mark.parametrize("hint", [0, 300])
@pytest.mark.parametrize("delta", [False, True])
def test_any_log_decay(hint, delta):
    """Factors that fp32 does not hold, of states that are zero or small enough, and states cleared first."""
    m = make(360, [70, 20, 5], 4, 2, 64, 64, delta)
    m["g"][:, 0] = -1e30
    m["g"][:, 1] = -300.0
    m["g"][2:, 2] = -0.5
    m["g"][1, 2] = 100.0                           # a state of zero, and one of 1e-30
    m["g"][70:90, 3] = 0.0
    m["g"][75, 3] = -math.inf                      # cleared, then a factor of e^95 with nothing written between
    m["g"][76, 3] = 95.0
    m["qkv"][:2, 2 * 2 * 64:2 * 2 * 64 + 4 * 64] = 0
    m["qkv"][75:77, 2 * 2 * 64:2 * 2 * 64 + 4 * 64] = 0
    m["pool"][0, 1, 2] *= 1e-30
    m["pool"][1, 1, 2] = 0
    if delta:
        m["beta"][75:77] = 0
        m["beta"][1, 2] = 0
    check(m, [0, 1, 2], [3, 4, 5], call(m, [0, 1, 2], [3, 4, 5], max_len=hint))

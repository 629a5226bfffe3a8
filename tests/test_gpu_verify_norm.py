"""dasc_verify_drafts against Python integers (equal), and dasc_block_norm against its formulas in
64 bits: every output within one rounding of its type (8 significant bits: 2^-8 bf16; 2^-11 fp16, relative) and the
fp32 chain before it (about ten roundings and sums of up to n terms: 2^-24 (16 + sqrt n) of the
terms that were added)."""

import math

import numpy as np
import pytest

import paper_2608_30386_amd as D
from oracle import operators as OO
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu


# ---- verification ---------------------------------------------------------------------------

def probabilities(gen, *shape, sharp=2.0):
    import torch

    return torch.softmax(torch.randn(shape, generator=gen) * sharp, -1)


def run_verify(target, draft, tokens, u, r, count, pad=0, **kw):
    import torch

    n, m1, V = target.shape
    def strided(x):                                    # rows `pad` apart, so of any alignment
        if x is None or not pad:
            return None if x is None else x.cuda()
        y = torch.full((*x.shape[:-1], V + pad), math.nan, dtype=x.dtype, device="cuda")
        y[..., :V] = x.cuda()
        return y[..., :V]
    out = torch.full((n, m1), 77, dtype=torch.int32, device="cuda")
    emitted = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    announce(f"verify n={n} m={m1 - 1} V={V} {target.dtype} draft={draft is not None}")
    D.dasc_verify_drafts(strided(target), tokens.cuda(), u.cuda(), r.cuda(), out, emitted,
                         draft=strided(draft), n_draft=None if count is None else count.cuda(), **kw)
    torch.cuda.synchronize()
    return out.cpu().numpy(), emitted.cpu().numpy()


def check_verify(target, draft, tokens, u, r, count, got):
    out, emitted = got
    n, m1, _ = target.shape
    tf = target.float().numpy()
    df = None if draft is None else draft.float().numpy()
    for i in range(n):
        k = m1 - 1 if count is None else min(int(count[i]), m1 - 1)
        toks, num = OO.verify(tf[i], None if df is None else df[i], tokens[i].numpy(), k, u[i].numpy(),
                              r[i].item())
        assert emitted[i] == num, (i, emitted[i], num)
        assert list(out[i]) == toks + [-1] * (m1 - len(toks)), (i, out[i], toks)


def verify_inputs(seed, n, m, V, dtype, with_draft, ragged):
    import torch

    gen = torch.Generator().manual_seed(seed)
    target = probabilities(gen, n, m + 1, V).to(dtype)
    near = torch.softmax(torch.log(target[:, :m].float() + 1e-9)
                         + 0.5 * torch.randn((n, m, V), generator=gen), -1).to(dtype)
    tokens = torch.multinomial(near.float().view(n * m, V) + 1e-12, 1, generator=gen).view(n, m).int() if m else \
        torch.zeros((n, 0), dtype=torch.int32)
    count = torch.randint(-1, m + 3, (n,), generator=gen).int() if ragged else None
    return (target, near if with_draft else None, tokens, torch.rand((n, m), generator=gen),
            torch.rand((n,), generator=gen), count)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,m,V", [(1, 4, 1000), (5, 3, 2048), (7, 0, 37), (3, 7, 2049), (2, 2, 1), (2, 1, 70001), (9, 1, 70001),
                                   (9, 300, 5)])
@pytest.mark.parametrize("with_draft", [False, True])
def test_verify(n, m, V, dtype, with_draft):
    import torch

    a = verify_inputs(n * 1000 + V, n, m, V, getattr(torch, dtype), with_draft, n > 1)
    check_verify(*a, run_verify(*a))
    check_verify(*a, run_verify(*a, pad=3))


def test_verify_many_rows_at_every_level():
    """One row drawn at many levels, the first and the last among them."""
    import torch

    n, V = 500, 3001
    gen = torch.Generator().manual_seed(3)
    row = probabilities(gen, 1, 1, V, sharp=4.0)
    target = row.expand(n, 1, V).contiguous()
    r = torch.linspace(0, 1, n)
    r[1], r[2], r[3], r[4] = 1 - 2.0 ** -24, 2.0 ** -24, 1.5, -0.5
    r[5] = math.nan
    a = (target, None, torch.zeros((n, 0), dtype=torch.int32), torch.zeros((n, 0)), r, None)
    check_verify(*a, run_verify(*a))


def test_verify_edges():
    """Rows with no weight, NaN, infinities, negative values, drafts outside the vocabulary, equal
    distributions, ties at the accept test, all the weight on the last token."""
    import torch

    V = 300
    gen = torch.Generator().manual_seed(4)
    base = probabilities(gen, 1, 1, V)[0, 0]
    zero = torch.zeros(V)
    last = zero.clone()
    last[-1] = 1.0
    odd = base.clone()
    odd[::5] = math.nan
    odd[1::5] = -1.0
    odd[2::50] = math.inf
    tiny = torch.full((V,), 2.0 ** -37)
    rows = [(base, base), (zero, base), (odd, base), (base, odd), (last, base), (base, last), (tiny, base),
            (zero, zero), (base, zero), (last, last), (base, torch.full((V,), math.nan))]
    target = torch.stack([torch.stack([p, p]) for p, _ in rows])
    draft = torch.stack([torch.stack([q]) for _, q in rows])
    n = len(rows)
    for tok, u in ((0, 0.999), (V - 1, 0.5), (-1, 0.0), (V, 0.0), (7, 0.0), (5, 1.0), (2, 0.25)):
        a = (target, draft, torch.full((n, 1), tok, dtype=torch.int32), torch.full((n, 1), u),
             torch.rand((n,), generator=gen), None)
        check_verify(*a, run_verify(*a))
        a = (target, None) + a[2:]
        check_verify(*a, run_verify(*a))


def test_verify_nothing_to_do_and_a_long_list():
    import torch

    e = torch.zeros((0, 3, 5), device="cuda")
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    D.dasc_verify_drafts(e, i(0, 2), torch.zeros((0, 2), device="cuda"), torch.zeros(0, device="cuda"),
                         i(0, 3), i(0))
    n, V = 40000, 6                                    # more requests than one grid row
    gen = torch.Generator().manual_seed(6)
    target = probabilities(gen, n, 2, V)
    tokens = torch.randint(0, V, (n, 1), generator=gen).int()
    a = (target, probabilities(gen, n, 1, V), tokens, torch.rand((n, 1), generator=gen),
         torch.rand((n,), generator=gen), None)
    out, emitted = run_verify(*a)
    some = list(range(0, n, 997)) + list(range(32760, 32780)) + [n - 1]
    check_verify(*(x if x is None else x[some] for x in a), (out[some], emitted[some]))


def test_verify_rows_beyond_32_bits():
    import torch

    V, m = 5000, 1
    stride = 2 ** 31 + 7
    flat = torch.zeros(stride + 2 * V, dtype=torch.bfloat16, device="cuda")
    a = verify_inputs(8, 2, m, V, torch.bfloat16, False, False)
    target = flat.as_strided((2, 2, V), (stride, V, 1))
    target.copy_(a[0].cuda())
    announce("verify with a request stride beyond 2^31")
    out = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    em = torch.zeros((2,), dtype=torch.int32, device="cuda")
    D.dasc_verify_drafts(target, a[2].cuda(), a[3].cuda(), a[4].cuda(), out, em)
    torch.cuda.synchronize()
    check_verify(*a, (out.cpu().numpy(), em.cpu().numpy()))


# ---- norms ------------------------------------------------------------------------------------

EPS = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}


def check_norm(kw, outs):
    """kw: the call's arguments on the CPU; outs: (x_out or None, h_out or None)."""
    d = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    xw, hw = OO.block_norm(d(kw["y"]), d(kw.get("gate")), kw.get("act", "none"), d(kw.get("w_post")),
                           d(kw.get("x")), kw.get("scale", 1.0), d(kw.get("channel_scale")), d(kw.get("w_pre")),
                           kw.get("eps", 1e-6))
    n = xw.shape[-1]
    chain = 2.0 ** -24 * (16 + math.sqrt(n))
    terms = np.abs(xw) + (np.abs(xw - d(kw["x"])) + np.abs(d(kw["x"])) if kw.get("x") is not None else 0)
    for name, got, want, size in (("x", outs[0], xw, terms), ("h", outs[1], hw, None)):
        if got is None:
            continue
        if size is None:
            rms = np.sqrt((xw * xw).mean(-1, keepdims=True) + kw.get("eps", 1e-6))
            size = np.abs(want) + terms / rms * np.abs(d(kw["w_pre"]))
        lim = EPS[str(got.dtype).split(".")[1]] * 1.01 * np.abs(want) + chain * size
        lim = lim + 2.0 ** -126 * 256                  # what fp32 holds below its smallest normal value
        if got.dtype.itemsize == 2 and "float16" == str(got.dtype).split(".")[1]:
            lim = lim + 2.0 ** -25                     # fp16's smallest steps
        err = np.abs(got.double().cpu().numpy() - want)
        assert np.all(err <= lim), (name, float((err / np.maximum(lim, 1e-300)).max()))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("dim", [1, 7, 16, 127, 128, 129, 512, 520, 1000, 2047, 2050, 4096, 5001, 8192, 9000, 16384, 20001,
                                 32768])
def test_norm_widths(dim, dtype):
    import torch

    dt = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(dim)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    rows = 5
    wide = rnd(rows, 2 * dim + 3).to(dt)
    kw = dict(y=rnd(rows, dim).to(dt), gate=wide[:, dim + 1:2 * dim + 1], act="silu", w_post=1 + 0.1 * rnd(dim),
              x=rnd(rows, dim), scale=0.7, channel_scale=rnd(dim), w_pre=1 + 0.1 * rnd(dim), eps=1e-5)
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    dev["gate"] = wide.cuda()[:, dim + 1:2 * dim + 1]
    xo = torch.full((rows, dim), 3.0, device="cuda")
    ho = torch.full((rows, dim + 5), 3.0, dtype=dt, device="cuda")
    announce(f"norm dim={dim} {dtype}")
    D.dasc_block_norm(**dev, x_out=xo, h_out=ho[:, 2:2 + dim])
    torch.cuda.synchronize()
    check_norm(kw, (xo, ho[:, 2:2 + dim]))
    assert torch.all(ho[:, :2] == 3.0) and torch.all(ho[:, 2 + dim:] == 3.0)


@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("post,res,pre,chan", [(1, 0, 0, 0), (0, 1, 1, 0), (1, 1, 0, 1), (1, 1, 1, 0), (0, 0, 1, 1)])
def test_norm_parts(gate, post, res, pre, chan):
    import torch

    gen = torch.Generator().manual_seed(9)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    bf = torch.bfloat16
    for rows, inner, dim in ((33, 3, 128), (17, 2, 96), (3, 1, 700)):
        shape = (rows, inner, dim)
        kw = dict(y=rnd(*shape).to(bf), scale=-1.5, act=gate)
        kw["gate"] = (3 * rnd(*shape)).to(bf) if gate != "none" else None
        kw["w_post"] = rnd(dim).to(bf) if post else None
        kw["x"] = rnd(*shape).to(bf) if res else None
        kw["channel_scale"] = rnd(dim).to(bf) if chan else None
        kw["w_pre"] = rnd(dim).to(bf) if pre else None
        dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
        xo = torch.empty(shape, dtype=bf, device="cuda")
        ho = torch.empty(shape, dtype=bf, device="cuda") if pre else None
        announce(f"norm parts {shape} gate={gate} post={post} res={res} pre={pre} chan={chan}")
        D.dasc_block_norm(**dev, x_out=xo, h_out=ho)
        torch.cuda.synchronize()
        check_norm(kw, (xo, ho))
        if pre:                                        # the outputs one at a time give the same bits
            h2 = torch.empty_like(ho)
            D.dasc_block_norm(**dev, h_out=h2)
            assert torch.equal(h2, ho)


def test_norm_in_place_and_repeated_rows():
    import torch

    gen = torch.Generator().manual_seed(10)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    for dim in (64, 3000, 10000):
        y, x, w = rnd(6, dim).bfloat16(), rnd(6, dim).bfloat16(), rnd(dim).bfloat16()
        kw = dict(y=y, x=x, w_post=w, w_pre=w, scale=0.5)
        xd, yd = x.cuda(), y.cuda()
        announce(f"norm in place dim={dim}")
        D.dasc_block_norm(yd, x=xd, w_post=w.cuda(), w_pre=w.cuda(), scale=0.5, x_out=xd, h_out=yd)
        torch.cuda.synchronize()
        check_norm(kw, (xd, yd))
        one = rnd(1, dim).bfloat16()                   # a gate row shared by all rows
        kw = dict(y=y, gate=one.expand(6, dim), act="sigmoid", w_post=w)
        xo = torch.empty((6, dim), dtype=torch.bfloat16, device="cuda")
        D.dasc_block_norm(y.cuda(), gate=one.cuda().expand(6, dim), act="sigmoid", w_post=w.cuda(), x_out=xo)
        torch.cuda.synchronize()
        check_norm(kw, (xo, None))


def test_norm_extremes():
    """Rows of zeros, very small and very large values, infinities in one row only, gates far out."""
    import torch

    y = torch.randn(6, 256, generator=torch.Generator().manual_seed(1))
    y[0] = 0
    y[1] *= 1e-18
    y[2] *= 1e15
    gate = torch.linspace(-200, 200, 256).expand(6, 256).contiguous()
    w = torch.ones(256)
    kw = dict(y=y, gate=gate, act="silu", w_post=w, eps=1e-6)
    xo = torch.empty((6, 256), device="cuda")
    D.dasc_block_norm(y.cuda(), gate=gate.cuda(), act="silu", w_post=w.cuda(), x_out=xo)
    torch.cuda.synchronize()
    check_norm(kw, (xo, None))
    bad = y.clone()
    bad[3, 7] = math.inf
    bad[4, 9] = math.nan
    x2 = torch.empty((6, 256), device="cuda")
    D.dasc_block_norm(bad.cuda(), gate=gate.cuda(), act="silu", w_post=w.cuda(), x_out=x2)
    torch.cuda.synchronize()
    keep = [0, 1, 2, 5]
    assert torch.equal(x2[keep], xo[keep])
    assert torch.isnan(x2[4]).all() and torch.isnan(x2[3, 7])


def test_norm_nothing_and_many_rows():
    import torch

    D.dasc_block_norm(torch.zeros((0, 8), device="cuda"), w_post=torch.ones(8, device="cuda"),
                      x_out=torch.zeros((0, 8), device="cuda"))
    rows = 70001
    y = torch.randn(rows, 24, generator=torch.Generator().manual_seed(2)).bfloat16()
    w = torch.ones(24).bfloat16()
    xo = torch.empty((rows, 24), dtype=torch.bfloat16, device="cuda")
    D.dasc_block_norm(y.cuda(), w_post=w.cuda(), x_out=xo)
    torch.cuda.synchronize()
    check_norm(dict(y=y, w_post=w), (xo, None))


def test_norm_rows_beyond_32_bits():
    import torch

    stride = 2 ** 31 + 5
    flat = torch.zeros(stride + 300, dtype=torch.bfloat16, device="cuda")
    y = flat.as_strided((2, 300), (stride, 1))
    src = torch.randn(2, 300, generator=torch.Generator().manual_seed(3)).bfloat16()
    y.copy_(src.cuda())
    w = torch.ones(300).bfloat16()
    announce("norm with a row stride beyond 2^31, in place")
    D.dasc_block_norm(y, w_post=w.cuda(), x_out=y)
    torch.cuda.synchronize()
    check_norm(dict(y=src, w_post=w), (y, None))

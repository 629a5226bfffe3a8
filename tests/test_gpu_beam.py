"""Selection of beams and moves of slots against their definitions (GPU).

Tokens, parents and slots have to be equal; scores are 64-bit values rounded to fp32, so they may differ from
the oracle's rounding by one step where 64-bit arithmetic of another order falls on the other side:
2^-23 of the value.  Moved slots are equal bit by bit.
"""

import numpy as np
import pytest

import paper_2608_30386_amd as D
from oracle import cache as OC
from tests.gpu_util import announce, dev_i32

pytestmark = pytest.mark.gpu


def select(logits, scores, n_out, slots=None, **over):
    import torch

    n = logits.shape[0]
    out = [torch.full((n, n_out), -7, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    D.dasc_beam_select(logits, scores, *out[:3], slots=slots, out_slots=out[3] if slots is not None else None, **over)
    torch.cuda.synchronize()
    return out


def check(logits, scores, n_out):
    import torch

    n, beams, _ = logits.shape
    slots = dev_i32(100 + np.random.default_rng(1).permutation(n * beams).reshape(n, beams))
    s, t, p, at = (x.cpu().numpy() for x in select(logits, scores, n_out, slots))
    x, start = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    for r in range(n):
        want = OC.beam_select(x[r], start[r], n_out)
        assert [w[1] for w in want] == t[r].tolist(), r
        assert [w[2] for w in want] == p[r].tolist(), r
        home = slots[r].tolist()
        assert [home[b] if b >= 0 else -1 for b in p[r]] == at[r].tolist()
        ws = np.array([w[0] for w in want])
        fin = np.isfinite(ws)
        assert (np.abs(s[r][fin] - ws[fin]) <= 2.0 ** -23 * np.abs(ws[fin])).all()
        assert (s[r][~fin] == -np.inf).all()


def rnd(*size, seed=0, dtype="float32", scale=3.0):
    import torch

    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(size, device="cuda", generator=g) * scale).to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,beams,vocab,n_out", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 17, 6), (1, 4, 4096, 4), (3, 2, 4097, 64),
                                                 (2, 64, 700, 64), (1, 5, 32001, 10), (5, 8, 8191, 16), (1, 2, 131071, 33)])
def test_select(n, beams, vocab, n_out, dtype):
    import torch

    announce(f"beam select n={n} beams={beams} vocab={vocab} n_out={n_out} {dtype}")
    check(rnd(n, beams, vocab, seed=vocab, dtype=dtype), -torch.rand(n, beams, device="cuda") * 4, n_out)


def test_ties_orders_and_equal_beams():
    import torch

    announce("beam select: ties")
    x = rnd(4, 4, 9000, seed=5).round()                    # few values, many ties
    x[0, :] = x[0, :1]                                     # equal beams
    x[1] = 0.0
    x[1, 2, ::2] = -0.0
    x[2] = torch.arange(9000, device="cuda") * 1e-3
    x[3] = -torch.arange(9000, device="cuda") * 1e-3
    check(x, torch.zeros(4, 4, device="cuda"), 16)
    y = rnd(1, 2, 20000, seed=6)
    y[0, 1] = y[0, 0].flip(0)
    check(y, torch.zeros(1, 2, device="cuda"), 64)
    # large values in one place of every lane's eight tokens, in few lanes, and in one run
    z = rnd(1, 3, 40000, seed=7)
    z[0, 0, ::8] += 50
    z[0, 1, 4096:4096 + 600] += 50
    z[0, 2, 8000:8003] += 50
    check(z, torch.zeros(1, 3, device="cuda"), 64)


def test_what_gives_no_candidate():
    import torch

    announce("beam select: infinities and NaN")
    inf, nan = float("inf"), float("nan")
    x = rnd(7, 3, 5000, seed=8)
    s = torch.zeros(7, 3, device="cuda")
    x[0, 1, 77] = nan
    x[1, 0, 4500] = inf
    x[2, 2] = -inf                                         # a row of nothing
    x[3] = -inf
    x[3, 1, 4321] = -2.0                                   # one candidate in all
    s[4, 0], s[4, 1] = -inf, nan
    s[5, 2] = inf
    x[6, :, 100:] = torch.finfo(torch.float32).min         # masked by the type's lowest value
    check(x, s, 12)
    s[:] = -inf
    check(x, s, 12)
    check(torch.full((2, 2, 300), -inf, device="cuda"), torch.zeros(2, 2, device="cuda"), 3)
    y = rnd(1, 2, 5000, seed=8)
    y[:, :, 64:] = torch.finfo(torch.float32).min
    y[:, :, :64] = -inf
    check(y, torch.zeros(1, 2, device="cuda"), 64)


def test_strided_rows_streams_graphs_and_one_workspace():
    import torch

    announce("beam select: strides, graph")
    wide = rnd(3, 4, 6003, seed=9)
    x, s = wide[:, 1:3, 3:6000], -torch.rand(3, 2, device="cuda")
    check(x, s, 5)
    assert D.dasc_beam_select_workspace_bytes(3, 2, 5997, 5) <= D.dasc_beam_select_workspace_bytes(4, 2, 6000, 5)
    ws = torch.empty(D.dasc_beam_select_workspace_bytes(4, 2, 6000, 5), dtype=torch.uint8, device="cuda")
    want = select(x, s, 5)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = select(x, s, 5, workspace=ws, stream=st)
    for a, b in zip(want[:3], got[:3]):
        assert torch.equal(a, b)
    out = [torch.empty_like(t) for t in want[:3]]
    run = lambda: D.dasc_beam_select(x, s, *out, workspace=ws)  # noqa: E731
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(3):
        wide.copy_(rnd(3, 4, 6003, seed=20 + i))
        g.replay()
        got = [t.clone() for t in out]
        for a, b in zip(select(x, s, 5)[:3], got):
            assert torch.equal(a, b)
    empty = torch.empty(0, 2, 10, device="cuda")
    select(empty, torch.empty(0, 2, device="cuda"), 4)


@pytest.mark.parametrize("m", [1, 4, 7, 8, 16, 23, 32, 64])
def test_moves_happen_at_once(m):
    import torch

    announce(f"move slots m={m}")
    rng = np.random.default_rng(m)
    groups, n = 3, 3 * m + 5
    pool = torch.randn(n, 1, 3, 4, 8, device="cuda")
    slots = rng.permutation(n)[:groups * m].reshape(groups, m)
    src = np.stack([rng.choice(s, m) for s in slots])      # a group's parents: any, several times
    dst = slots.copy()
    if m > 3:
        src[0, 1], dst[1, 2] = -1, n                       # left out
    want = OC.move_slots(pool.cpu().numpy(), src, dst)
    wide = torch.zeros(groups, m + 3, dtype=torch.int32, device="cuda")
    wide[:, :m] = dev_i32(src)
    D.dasc_move_slots(pool, wide[:, :m], dev_i32(dst))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(pool.cpu().numpy().view(np.uint32), want.view(np.uint32))


def test_moves_of_pages_and_far_slots():
    import torch

    announce("move slots: strided pages, offsets beyond 32 bits")
    pages = torch.randint(0, 30000, (40, 2, 16, 3, 8), dtype=torch.int16, device="cuda")
    want = OC.move_slots(pages[:, 1].cpu().numpy(), [3, 5], [5, 39])
    left = pages[:, 0].clone()
    D.dasc_move_slots(pages[:, 1], dev_i32([3, 5]), dev_i32([5, 39]))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(pages[:, 1].cpu().numpy(), want)
    assert torch.equal(pages[:, 0], left)
    big = torch.zeros(9, 2 ** 29 + 16, dtype=torch.uint8, device="cuda")
    big[0] = 7
    big[8, -1] = 9
    D.dasc_move_slots(big, dev_i32([0, 8]), dev_i32([8, 0]))
    torch.cuda.synchronize()
    assert int(big[8].min()) == 7 and int(big[0].max()) == 9 and int(big[0, -1]) == 9 and int(big[0, 0]) == 0
    D.dasc_move_slots(big, dev_i32([]).view(0, 4), dev_i32([]).view(0, 4))


def test_a_beam_step():
    """Select, then move the states of the parents to the beams' slots, in place."""
    import torch

    announce("beam step")
    n, B, V = 3, 4, 900
    x, s = rnd(n, B, V, seed=11), -torch.rand(n, B, device="cuda")
    slots = dev_i32(np.random.default_rng(2).permutation(n * B + 2)[:n * B].reshape(n, B))
    pool = torch.randn(n * B + 2, 2, 2, 16, 16, device="cuda")
    _, _, parents, src = select(x, s, 2 * B, slots)
    home = slots.cpu().numpy()
    from_ = np.take_along_axis(home, parents[:, :B].cpu().numpy(), 1)
    want = OC.move_slots(pool.cpu().numpy(), from_, home)
    D.dasc_move_slots(pool, src[:, :B], slots)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(pool.cpu().numpy().view(np.uint32), want.view(np.uint32))


def test_more_rows_than_a_launch_takes():
    import torch

    announce("beam select: 40000 requests")
    n, vocab = 40000, 20
    x, s = rnd(n, 1, vocab, seed=12), -torch.rand(n, 1, device="cuda")
    top, token, parent, _ = select(x, s, 3)
    want, at = torch.sort(s.double()[..., None] + torch.log_softmax(x.double(), -1), dim=-1, descending=True, stable=True)
    assert torch.equal(token, at[:, 0, :3].int()) and (parent == 0).all()
    assert ((top - want[:, 0, :3]).abs() <= 2.0 ** -23 * want[:, 0, :3].abs()).all()


def test_moves_of_many_groups():
    import torch

    announce("move slots: 3000 groups")
    groups, m = 3000, 2
    pool = torch.randn(groups * m, 4, device="cuda")
    slots = np.random.default_rng(3).permutation(groups * m).reshape(groups, m)
    want = OC.move_slots(pool.cpu().numpy(), slots[:, ::-1], slots)
    D.dasc_move_slots(pool, dev_i32(slots[:, ::-1].copy()), dev_i32(slots))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(pool.cpu().numpy(), want)

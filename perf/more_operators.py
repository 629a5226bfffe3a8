"""Workloads that time the operators of a hybrid model's full-attention layers and of its beams.

Three operators: the append of rotated keys and values to a paged cache, the attention of new
tokens over that cache, and the selection of beams with the reordering of their recurrent states.
A case is one call (a beam case: the selection and the states' move).  State shapes are those of
`workloads/synth.py` (Qwen3-Next-shaped GDN layers of 32 heads of 128 x 128) and of the tests;
attention heads, pages and vocabularies are generic.

`own` chooses what `run` does: the plain form (elementary torch operations in 32 bits, angles and
log-sums in 64) or the library's calls.
"""

import math
import random

import torch

own = False


def listed():
    grouped = dict(kind="attn", Hq=32, Hkv=8, d=128, page=16, heads_first=False, dtype="bfloat16",
                   causal=True, window=0, lse=False)
    wide = dict(grouped, Hq=16, Hkv=2, d=256)
    return [
        # four decoded tokens, a quarter of each head rotated: the smallest call, all latency
        dict(name="append_token", kind="append", N=4, Hq=16, Hkv=2, d=256, rot=64, page=16,
             heads_first=False, axes=1, adjacent=False, dtype="bfloat16", padded=False),
        # a prompt's chunk of 8192 tokens, whole heads rotated
        dict(name="append_prompt", kind="append", N=8192, Hq=32, Hkv=8, d=128, rot=128, page=16,
             heads_first=False, axes=1, adjacent=False, dtype="bfloat16", padded=False),
        # image and text tokens at positions of three axes, a padded batch of an odd number of rows
        dict(name="append_axes", kind="append", N=3001, Hq=28, Hkv=4, d=128, rot=128, page=64,
             heads_first=True, axes=3, adjacent=True, dtype="float16", padded=True),
        # one token of one request over about a thousand keys
        dict(wide, name="attn_token_one", n=1, new=1, kv=1027, ragged=False),
        # a decode batch of 64 requests whose contexts run from 1.5 to 10 thousand tokens
        dict(grouped, name="attn_token_batch", n=64, new=1, kv=6000, ragged=True),
        # 48 requests score four drafts each, with the log-sums of their rows
        dict(wide, name="attn_drafts", n=48, new=5, kv=2500, ragged=True, lse=True),
        # a chunk of 2048 new tokens of one long prompt
        dict(wide, name="attn_chunk", n=1, new=2048, kv=30011, ragged=False),
        # eight whole prompts of 300 to 2000 tokens, nothing cached before
        dict(grouped, name="attn_prompts", n=8, new=1211, kv=0, ragged=True),
        # small heads without groups, a sliding window, pages of an odd size, 4097 tokens
        dict(grouped, name="attn_window", n=1, new=4097, kv=0, ragged=False, Hq=16, Hkv=16, d=64,
             page=24, heads_first=True, dtype="float16", window=1000),
        # one request of four beams, fp32 logits, states of 16 heads of 64 x 64
        dict(name="beam_one", kind="beam", n=1, beams=4, out=4, vocab=32000, dtype="float32", H=16, dk=64),
        # 16 requests of eight beams, an odd vocabulary in bf16, states of a layer of 32 heads of 128 x 128
        dict(name="beam_batch", kind="beam", n=16, beams=8, out=16, vocab=131071, dtype="bfloat16", H=32,
             dk=128),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: head layouts of a layer or of a tensor-parallel rank's share,
    batches, lengths, pages and vocabularies log-uniform, odd ones among them."""
    kind = rng.choice(["append", "token", "token", "drafts", "chunk", "prompts", "beam"])
    if kind == "beam":
        beams = rng.randint(2, 16)
        return dict(kind="beam", n=_logint(rng, 1, 16), beams=beams, out=rng.choice([beams, 2 * beams]),
                    vocab=_logint(rng, 1000, 131071), dtype=rng.choice(["float32", "bfloat16", "float16"]),
                    H=rng.choice([4, 8, 16, 32]), dk=rng.choice([64, 128]))
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    Hkv = rng.choice([h for h in (1, 2, 4, 8, 16) if h * group <= 32])
    c = dict(Hq=Hkv * group, Hkv=Hkv, d=rng.choice([64, 96, 128, 128, 256]),
             page=rng.choice([1, 8, 16, 16, 24, 64, 100, 256]), heads_first=rng.random() < 0.4,
             dtype=rng.choice(["bfloat16", "bfloat16", "float16"]))
    if kind == "append":
        rot = rng.choice([c["d"], c["d"], c["d"] // 2, c["d"] // 4])
        return dict(c, kind="append", N=_logint(rng, 1, 8192), rot=rot, axes=rng.choice([1, 1, 2, 3]),
                    adjacent=rng.random() < 0.5, padded=rng.random() < 0.3)
    c.update(kind="attn", causal=True, window=0, lse=rng.random() < 0.3)
    if kind == "token":
        kv = _logint(rng, 1, 16000)
        n = _logint(rng, 1, max(1, min(64, int(1.2e9 / (4 * kv * c["Hkv"] * c["d"])))))
        return dict(c, n=n, new=1, kv=kv, ragged=n > 1)
    if kind == "drafts":
        kv = _logint(rng, 50, 8000)
        n = _logint(rng, 1, max(1, min(48, 120000 // kv)))
        return dict(c, n=n, new=rng.randint(2, 8), kv=kv, ragged=n > 1, causal=rng.random() < 0.8)
    if rng.random() < 0.25:
        c["window"] = _logint(rng, 16, 2000)
    if kind == "chunk":
        return dict(c, n=1, new=_logint(rng, 20, 2048), kv=_logint(rng, 500, 20000), ragged=False)
    new = _logint(rng, 20, 4097)
    n = _logint(rng, 1, max(1, min(12, 6000 // new)))
    return dict(c, n=n, new=new, kv=0, ragged=n > 1)


# ---- inputs ---------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    s = {"append": _prepare_append, "attn": _prepare_attn, "beam": _prepare_beam}[case["kind"]](case, seed)
    if own:
        import paper_2608_30386_amd as D
        s["D"] = D
    return s


def _pool(c, n_pages, gen, dt):
    """Keys and values of a cache's pages [n_pages, page, Hkv, d], tokens or heads first in memory."""
    both = []
    for _ in range(2):
        if c["heads_first"]:
            x = torch.randn((n_pages, c["Hkv"], c["page"], c["d"]), device="cuda", generator=gen).to(dt)
            both.append(x.transpose(1, 2))
        else:
            both.append(torch.randn((n_pages, c["page"], c["Hkv"], c["d"]), device="cuda", generator=gen).to(dt))
    return both


def _prepare_append(c, seed):
    gen = _gen(seed)
    N, Hq, Hkv, d, page = c["N"], c["Hq"], c["Hkv"], c["d"], c["page"]
    dt = getattr(torch, c["dtype"])
    # q, k and v are slices of one projection's output
    qkv = torch.randn((N, (Hq + 2 * Hkv) * d), device="cuda", generator=gen).to(dt)
    q = qkv[:, :Hq * d].view(N, Hq, d)
    k = qkv[:, Hq * d:(Hq + Hkv) * d].view(N, Hkv, d)
    v = qkv[:, (Hq + Hkv) * d:].view(N, Hkv, d)
    n_pages = -(-N // page) + 2
    kc, vc = _pool(c, n_pages, gen, dt)
    # the tokens' pages in random order; page 0 is no request's
    order = 1 + torch.randperm(n_pages - 1, device="cuda", generator=gen)
    t = torch.arange(N, device="cuda")
    slots = order[t // page] * page + t % page
    if c["padded"]:                        # rows of the batch that belong to no request
        slots = torch.where(t % 17 == 16, -1, slots)
    start = int(random.Random(seed).uniform(0, 200000))
    pos = (start + t)[:, None].repeat(1, c["axes"])
    if c["axes"] > 1:                      # height and width on a grid of 32 columns
        pos[:, 1] = start + t // 32
        pos[:, -1] = start + t % 32
    half = c["rot"] // 2
    inv_freq = (1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
    axis = (torch.arange(half, device="cuda") * c["axes"] // half).int() if c["axes"] > 1 else None
    return dict(c=c, q=q, k=k, v=v, kc=kc, vc=vc, slots=slots, pos=pos.int(), inv_freq=inv_freq, axis=axis,
                q_out=torch.empty((N, Hq, d), dtype=dt, device="cuda"))


def _lengths(c):
    """New and cached tokens of each request: the same for every seed."""
    n = c["n"]
    if not c["ragged"]:
        return [c["new"]] * n, [c["kv"]] * n
    r = random.Random(n * 1000003 + c["new"] * 1009 + c["kv"])
    part = [r.uniform(0.25, 1.7) for _ in range(n)]
    old = [int(c["kv"] * x) for x in part]
    new = [c["new"]] * n if c["new"] <= 8 else [max(1, int(c["new"] * x)) for x in part]
    return new, old


def _prepare_attn(c, seed):
    gen = _gen(seed)
    n, Hq, Hkv, d, page = c["n"], c["Hq"], c["Hkv"], c["d"], c["page"]
    dt = getattr(torch, c["dtype"])
    new, old = _lengths(c)
    kv = [a + b for a, b in zip(new, old)]
    need = [-(-x // page) for x in kv]
    width = max(need)
    kc, vc = _pool(c, sum(need) + 1, gen, dt)
    order = torch.randperm(sum(need) + 1, device="cuda", generator=gen).int()
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    N = sum(new)
    cu = torch.tensor([0] + [sum(new[:i + 1]) for i in range(n)], dtype=torch.int32, device="cuda")
    s = dict(c=c, kc=kc, vc=vc, table=table, cu=cu, kv=torch.tensor(kv, dtype=torch.int32, device="cuda"),
             q=(torch.randn((N, Hq, d), device="cuda", generator=gen) * 1.5).to(dt),
             o=torch.empty((N, Hq, d), dtype=dt, device="cuda"), max_new=max(new), max_kv=max(kv),
             lse=torch.empty((N, Hq), device="cuda") if c["lse"] else None, scale=d ** -0.5)
    if own:
        import paper_2608_30386_amd as D
        s["ws"] = torch.empty(max(1, D.dasc_cache_attn_workspace_bytes(n, N, Hq, Hkv, d, max(new), max(kv))),
                              dtype=torch.uint8, device="cuda")
    return s


def _prepare_beam(c, seed):
    gen = _gen(seed)
    n, B, V = c["n"], c["beams"], c["vocab"]
    dt = getattr(torch, c["dtype"])
    # logits as a head leaves them: a few tokens stand out
    logits = (torch.randn((n, B, V), device="cuda", generator=gen) * 3).to(dt)
    scores = -5 * torch.rand((n, B), device="cuda", generator=gen)
    # two sets of slots that a request's beams change between from step to step
    slots = torch.randperm(2 * n * B, device="cuda", generator=gen).int().view(2, n, B)
    pool = torch.randn((2 * n * B, 1, c["H"], c["dk"], c["dk"]), device="cuda", generator=gen) * 0.05
    e = lambda t: torch.empty((n, c["out"]), dtype=t, device="cuda")  # noqa: E731
    s = dict(c=c, logits=logits, scores=scores, now=slots[0].contiguous(), next=slots[1].contiguous(), pool=pool,
             out_scores=e(torch.float32), tokens=e(torch.int32), parents=e(torch.int32), src=e(torch.int32))
    if own:
        import paper_2608_30386_amd as D
        s["ws"] = torch.empty(max(1, D.dasc_beam_select_workspace_bytes(n, B, V, c["out"])), dtype=torch.uint8,
                              device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(s):
    return {"append": _run_append, "attn": _run_attn, "beam": _run_beam}[s["c"]["kind"]](s)


def _run_append(s):
    c = s["c"]
    if own:
        s["D"].dasc_cache_append(s["kc"], s["vc"], s["slots"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], pos=s["pos"],
                                 inv_freq=s["inv_freq"], pair_axis=s["axis"], adjacent=c["adjacent"])
        return {"q": s["q_out"], "k": s["kc"], "v": s["vc"]}
    half, page, dt = c["rot"] // 2, c["page"], s["q"].dtype
    pos = s["pos"][:, :1] if s["axis"] is None else s["pos"][:, s["axis"].long()]
    angle = (pos.double() * s["inv_freq"].double())[:, None]                  # [N, 1, half]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def rotate(x):
        x = x.float()
        r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["adjacent"]:
            a, b = r[..., 0::2], r[..., 1::2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([y, rest], -1).to(dt)

    at = s["slots"].clamp_min(0)
    live = (s["slots"] >= 0)[:, None, None]
    for cache, x in ((s["kc"], rotate(s["k"])), (s["vc"], s["v"])):
        cache[at // page, at % page] = torch.where(live, x, cache[at // page, at % page])
    return {"q": rotate(s["q"]), "k": s["kc"], "v": s["vc"]}


def _run_attn(s):
    c = s["c"]
    if own:
        s["D"].dasc_cache_attn(s["kc"], s["vc"], s["table"], s["kv"], s["q"], s["o"], s["cu"], s["max_new"],
                               max_kv=s["max_kv"], scale=s["scale"], causal=c["causal"], window=c["window"],
                               lse=s["lse"], workspace=s["ws"])
        return {"o": s["o"], **({"lse": s["lse"]} if c["lse"] else {})}
    n, Hkv, d, page, G = c["n"], c["Hkv"], c["d"], c["page"], c["Hq"] // c["Hkv"]
    L, K, dev, dt = s["max_new"], s["max_kv"], s["q"].device, s["q"].dtype
    t, p = torch.arange(L, device=dev), torch.arange(K, device=dev)
    count = s["cu"][1:] - s["cu"][:-1]
    live = t < count[:, None]                                                 # [n, L]
    q = s["q"][torch.where(live, s["cu"][:-1, None] + t, 0)].float().view(n, L, Hkv, G, d)
    q = q.permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * L, d)
    pages = s["table"][:, p // page].long().clamp_min(0)                      # [n, K]
    k = s["kc"][pages, p % page].float().permute(0, 2, 3, 1)                  # [n, Hkv, d, K]
    v = s["vc"][pages, p % page].float().transpose(1, 2)                      # [n, Hkv, K, d]
    x = ((q @ k) * s["scale"]).view(n, Hkv, G, L, K)
    here = (s["kv"] - count)[:, None] + t                                     # [n, L]: a token's own position
    seen = (p < s["kv"][:, None])[:, None, :].expand(n, L, K)
    if c["causal"]:
        seen = seen & (p <= here[..., None])
    if c["window"]:
        seen = seen & (p > here[..., None] - c["window"])
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(n, Hkv, G * L, K) @ v).view(n, Hkv, G, L, d) / torch.where(total > 0, total, 1.0)
    out = {"o": o.permute(0, 3, 1, 2, 4)[live].reshape(-1, c["Hq"], d).to(dt)}
    if c["lse"]:
        out["lse"] = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2)[live].reshape(-1, c["Hq"])
    return out


def _run_beam(s):
    c, n, B, out = s["c"], s["c"]["n"], s["c"]["beams"], s["c"]["out"]
    if own:
        s["D"].dasc_beam_select(s["logits"], s["scores"], s["out_scores"], s["tokens"], s["parents"], slots=s["now"],
                                out_slots=s["src"], workspace=s["ws"])
        s["D"].dasc_move_slots(s["pool"], s["src"][:, :B], s["next"])
        return {"scores": s["out_scores"], "tokens": s["tokens"], "parents": s["parents"], "pool": s["pool"]}
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True).double()
    lse = top[..., 0] + torch.log(torch.exp(x.double() - top).sum(-1))        # [n, B]
    # a beam's best tokens: one whole number orders by logit, then by the lower token
    bits = x.view(torch.int32)
    bits = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    key = (bits << 32) | (0xFFFFFFFF - torch.arange(c["vocab"], device=x.device))
    m = min(out, c["vocab"])
    token = 0xFFFFFFFF - (torch.topk(key, m, -1).values & 0xFFFFFFFF)         # [n, B, m]
    score = s["scores"].double()[..., None] + (x.gather(-1, token).double() - lse[..., None])
    # parents ascending and tokens of equal score ascending: a stable sort keeps the lowest index first
    score, at = torch.sort(score.view(n, B * m), dim=-1, descending=True, stable=True)
    at = at[:, :out]
    parents = at // m
    src = s["now"].gather(1, parents)[:, :B].long()
    s["pool"][s["next"].long()] = s["pool"][src]
    return {"scores": score[:, :out].float(), "tokens": token.view(n, B * m).gather(1, at).int(),
            "parents": parents.int(), "pool": s["pool"]}


# ---- what a pass cannot do without --------------------------------------------------------------

def _pairs(new, kv, causal, window):
    """(query, key) pairs of a request that its mask leaves."""
    total = 0
    for t in range(new):
        here = kv - new + t
        hi = min(kv, here + 1) if causal else kv
        total += max(0, hi - (max(0, here - window + 1) if window else 0))
    return total


def work(case):
    c = case
    if c["kind"] == "append":
        n = c["N"] - (c["N"] // 17 if c["padded"] else 0)
        moved = c["d"] * (c["N"] * c["Hq"] + 2 * n * c["Hkv"])
        return {"bytes": 4 * moved + c["N"] * (8 + 4 * c["axes"]),
                "flops": 3 * c["rot"] * (c["N"] * c["Hq"] + n * c["Hkv"])}
    if c["kind"] == "attn":
        new, old = _lengths(c)
        kv = [a + b for a, b in zip(new, old)]
        reach = [min(b, a + c["window"] - 1) if c["window"] else b for a, b in zip(new, kv)]
        b = 4 * c["d"] * (sum(new) * c["Hq"] + sum(reach) * c["Hkv"]) + 4 * sum(-(-x // c["page"]) for x in reach)
        if c["lse"]:
            b += 4 * sum(new) * c["Hq"]
        pairs = sum(_pairs(x, y, c["causal"], c["window"]) for x, y in zip(new, kv))
        return {"bytes": b, "flops": 4 * c["d"] * c["Hq"] * pairs}
    e = 4 if c["dtype"] == "float32" else 2
    rows = c["n"] * c["beams"]
    state = 4 * c["H"] * c["dk"] * c["dk"]
    # of eight parents drawn from eight beams about half are distinct
    return {"bytes": rows * c["vocab"] * e + rows * state * 1.5 + 20 * c["n"] * c["out"], "flops": 4 * rows * c["vocab"]}


# ---- the same in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "beam": _exact_beam}[case["kind"]](s)


def _exact_append(s):
    """Each pair as a complex number, turned by its angle."""
    c = s["c"]
    page, half, rot = c["page"], c["rot"] // 2, c["rot"]
    axis = torch.zeros(half, dtype=torch.long, device="cuda") if s["axis"] is None else s["axis"].long()
    angle = s["pos"].double().index_select(1, axis) * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotated(x):
        y = x.double().clone()
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if c["adjacent"] else (slice(0, half), slice(half, rot))
        z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    on = torch.nonzero(s["slots"] >= 0)[:, 0]
    at = s["slots"][on]
    kc, vc = s["kc"].double(), s["vc"].double()
    kc[at // page, at % page] = rotated(s["k"])[on]
    vc[at // page, at % page] = s["v"].double()[on]
    return {"q": rotated(s["q"]), "k": kc, "v": vc}


def _exact_attn(s):
    """A request and key head at a time, from the softmax's definition."""
    c = s["c"]
    page, G, cu, kv = c["page"], c["Hq"] // c["Hkv"], s["cu"].tolist(), s["kv"].tolist()
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for i in range(c["n"]):
        rows = slice(cu[i], cu[i + 1])
        p = torch.arange(kv[i], device="cuda")
        at = torch.arange(cu[i + 1] - cu[i], device="cuda") + kv[i] - (cu[i + 1] - cu[i])
        far = at[:, None] - p                                                 # how far back a key lies
        hide = torch.zeros_like(far, dtype=torch.bool)
        if c["causal"]:
            hide |= far < 0
        if c["window"]:
            hide |= far >= c["window"]
        pages = s["table"][i].long()[p // page]
        for h in range(c["Hkv"]):
            k, v = s["kc"][pages, p % page, h].double(), s["vc"][pages, p % page, h].double()
            for g in range(h * G, (h + 1) * G):
                x = s["scale"] * (s["q"][rows, g].double() @ k.t().contiguous())
                x[hide] = -math.inf
                lse[rows, g] = torch.logsumexp(x, -1)
                o[rows, g] = torch.softmax(x, -1) @ v
    return {"o": o, **({"lse": lse} if c["lse"] else {})}


def _exact_beam(s):
    c, n, B, out = s["c"], s["c"]["n"], s["c"]["beams"], s["c"]["out"]
    scores = s["scores"].double()[..., None] + torch.log_softmax(s["logits"].double(), -1)
    best, parents = [], []
    for i in range(n):                       # tokens whole numbers; the floats go by them
        x, at = torch.sort(scores[i].reshape(-1), descending=True, stable=True)
        best.append(x[:out])
        parents.append(at[:out] // c["vocab"])
    src = s["now"].gather(1, torch.stack(parents))[:, :B].long()
    pool = s["pool"].double()
    pool[s["next"].long()] = pool[src]
    return {"scores": torch.stack(best), "tokens": None, "parents": None, "pool": pool}

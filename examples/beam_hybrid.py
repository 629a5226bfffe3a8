"""Beam search on a small hybrid stack: GDN layers with recurrent states, attention layers with a paged cache.

Random weights, synthetic tokens; one GPU.  The steps and the calls that carry them:

  prompt      a GDN layer: dasc_linear_attn into each request's first slot; an attention layer:
              dasc_cache_append of its rotated keys and values, dasc_cache_attn over them
  fork        dasc_move_slots: the first beam's states and last, partly filled pages to the others' (whole
              pages of the prompt are shared)
  step        the same layers over one token of every beam, dasc_beam_select of the best continuations,
              dasc_move_slots of states and last pages after their parents, all at once and in place

The norms around the layers are dasc_block_norm.  A beam's pages before its last one are never written
again, so beams may share them: a reordering copies the table's rows and one page a layer.

    python examples/beam_hybrid.py --requests 4 --beams 4 --steps 16
"""

from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_30386_amd as D  # noqa: E402

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=I32, device="cuda")


class Hybrid:
    """`layers` blocks, every `every`-th of them attention, between an embedding and a head; weights from `seed`."""

    def __init__(self, layers=4, every=2, heads=4, dk=64, q_heads=8, kv_heads=2, head_dim=64, width=256, vocab=1024,
                 seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)

        def w(*size):
            return (torch.randn(size, generator=gen, device="cuda") / size[0] ** 0.5).to(BF16)

        self.kinds = ["attn" if i % every == every - 1 else "gdn" for i in range(layers)]
        n_gdn = self.kinds.count("gdn")
        self.shape = D.Shape("gdn", n_gdn, heads, heads, dk, dk)
        self.q_heads, self.kv_heads, self.d, self.vocab = q_heads, kv_heads, head_dim, vocab
        self.n_attn = layers - n_gdn
        self.embed = torch.randn(vocab, width, generator=gen, device="cuda").to(BF16)
        self.head = w(width, vocab)
        self.norm = torch.ones(width, device="cuda", dtype=BF16)
        self.half = torch.full((width,), 0.5, device="cuda", dtype=BF16)
        self.inv_freq = (1e4 ** (-torch.arange(head_dim // 4) / (head_dim // 4))).float().cuda()   # half of a head
        self.decay = torch.tensor(-np.geomspace(1e-3, 0.5, heads), device="cuda", dtype=F32)
        self.blocks = []
        for kind in self.kinds:
            if kind == "gdn":
                self.blocks.append(dict(x=w(width, 3 * heads * dk), b=w(width, heads), o=w(heads * dk, width)))
            else:
                self.blocks.append(dict(x=w(width, (q_heads + 2 * kv_heads) * head_dim), o=w(q_heads * head_dim, width)))

    def forward(self, tokens, pos, cu, max_len, states, slots, cache, table, kv_lens, at, rows):
        """Logits after the rows named by `rows`.  cache: [n_pages, attention layers, k or v, page, heads, d]."""
        s, n = self.shape, tokens.numel()
        x = self.embed[tokens]
        h = torch.empty_like(x)
        D.dasc_block_norm(x, w_post=self.norm, x_out=h)
        gdn = attn = 0
        for kind, b in zip(self.kinds, self.blocks):
            y = h @ b["x"]
            if kind == "gdn":
                q, k, v = y.view(n, 3, s.n_heads, s.dk).unbind(1)
                q, k = (F.normalize(t.float(), dim=-1).to(BF16) for t in (q, k))
                o = torch.empty(n, s.n_heads, s.dv, dtype=BF16, device="cuda")
                D.dasc_linear_attn(s, gdn, states, slots, slots, q, k, v, self.decay.expand(n, s.n_heads), o, cu, max_len,
                                   beta=torch.sigmoid((h @ b["b"]).float()), scale=s.dk ** -0.5)
                gdn += 1
            else:
                q, k, v = y.view(n, -1, self.d).split([self.q_heads, self.kv_heads, self.kv_heads], 1)
                kc, vc = cache[:, attn, 0], cache[:, attn, 1]
                o = torch.empty(n, self.q_heads, self.d, dtype=BF16, device="cuda")
                qr = torch.empty_like(o)
                D.dasc_cache_append(kc, vc, at, k, v, q=q, q_out=qr, pos=pos, inv_freq=self.inv_freq)
                D.dasc_cache_attn(kc, vc, table, kv_lens, qr, o, cu, max_len)
                attn += 1
            D.dasc_block_norm(o.view(n, -1) @ b["o"], w_post=self.half, x=x, w_pre=self.norm, x_out=x, h_out=h)
        return (h[rows] @ self.head).float()


def search(model, prompts, beams=4, steps=16, page=16):
    """The beams of every prompt (a list of tensors of tokens): tokens [n, beams, steps] and scores [n, beams], best
    first."""
    n, s = len(prompts), model.shape
    lens = np.array([len(p) for p in prompts])
    width = -(-int(lens.max() + steps) // page)
    # pages: a prompt's whole ones once, then for every beam those from the prompt's end on
    shared = lens // page
    n_pages = int(shared.sum()) + n * beams * (width + 1)
    order = np.random.default_rng(0).permutation(n_pages)
    table = np.full((n, beams, width), -1)
    free = 0
    for r in range(n):
        table[r, :, :shared[r]] = order[free:free + shared[r]]
        free += shared[r]
        own = beams * (width - shared[r])
        table[r, :, shared[r]:] = order[free:free + own].reshape(beams, -1)
        free += own
    cache = torch.zeros(n_pages, model.n_attn, 2, page, model.kv_heads, model.d, dtype=BF16, device="cuda")
    states = torch.empty(n * beams, s.n_layers, s.n_heads, s.dk, s.dv, device="cuda")
    slots = torch.arange(n * beams, dtype=I32, device="cuda").view(n, beams)

    # the prompts, on each request's first beam
    tokens = torch.cat(list(prompts))
    pos = torch.cat([torch.arange(k, device="cuda") for k in lens])
    cu = np.concatenate([[0], np.cumsum(lens)])
    req = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(lens, device="cuda"))
    pages = torch.tensor(table, device="cuda")
    at = pages[req, 0, pos // page] * page + pos % page
    states.zero_()
    logits = model.forward(tokens, pos.int(), i32(cu), int(lens.max()), states, slots[:, 0].contiguous(), cache,
                           pages[:, 0].int().contiguous(), i32(lens), at, torch.tensor(cu[1:] - 1, device="cuda"))
    last = torch.tensor(lens // page, device="cuda")               # the page that grows
    rows = torch.arange(n, device="cuda")
    D.dasc_move_slots(states, slots[:, :1].expand(n, beams).contiguous(), slots)
    D.dasc_move_slots(cache, pages[rows, :1, last].expand(n, beams).int().contiguous(), pages[rows, :, last].int())

    scores = torch.full((n, beams), -float("inf"), device="cuda")
    scores[:, 0] = 0.0                                              # one beam is in use
    best = lambda t: torch.empty(n, beams, dtype=t, device="cuda")  # noqa: E731
    out = torch.empty(n, beams, 0, dtype=I32, device="cuda")
    logits = logits.view(n, 1, -1).expand(n, beams, model.vocab).contiguous()
    length = torch.tensor(lens, device="cuda")
    one = i32(np.arange(n * beams + 1))
    for step in range(steps):
        top, token, parent, src = best(F32), best(I32), best(I32), best(I32)
        D.dasc_beam_select(logits, scores, top, token, parent, slots=slots, out_slots=src)
        scores = top
        who = parent.long()
        out = torch.cat([out.gather(1, who[..., None].expand(-1, -1, step)), token[..., None]], 2)
        if step + 1 == steps:
            break
        # states and growing pages go after their parents, in place; the pages before are shared by the table
        D.dasc_move_slots(states, src, slots)
        grow = pages[rows, :, length // page].int()
        D.dasc_move_slots(cache, grow.gather(1, who), grow)
        past = torch.arange(width, device="cuda") < (length // page)[:, None, None]
        pages = torch.where(past, pages.gather(1, who[..., None].expand(-1, -1, width)), pages)
        p = length[:, None].expand(n, beams)
        at = pages.gather(2, (p // page)[..., None])[..., 0] * page + p % page
        length = length + 1
        logits = model.forward(token.reshape(-1).long(), p.reshape(-1).int(), one, 1, states, slots.view(-1), cache,
                               pages.view(n * beams, width).int(), length.repeat_interleave(beams).int(), at.reshape(-1),
                               slice(None)).view(n, beams, -1)
    return out, scores


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    model = Hybrid(layers=a.layers)
    gen = torch.Generator("cuda").manual_seed(1)
    prompts = [torch.randint(model.vocab, (20 + 37 * i,), generator=gen, device="cuda") for i in range(a.requests)]
    search(model, prompts, a.beams, 2)                             # the first calls load the kernels
    torch.cuda.synchronize()
    t = time.perf_counter()
    out, scores = search(model, prompts, a.beams, a.steps)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"{a.requests} requests, {a.beams} beams, {a.steps} steps: {1e3 * t:.1f} ms; best scores "
          + " ".join(f"{x:.2f}" for x in scores[:, 0].tolist()))


if __name__ == "__main__":
    main()

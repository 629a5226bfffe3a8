"""Speculative serving of a small GDN stack: a prefix hit, prompts, drafts, verification, commit.

Random weights, synthetic tokens; one GPU.  The steps and the calls that carry them:

  prefix      dasc_linear_attn over the shared prefix (chunked form), dasc_pack of its state
  hit         dasc_restore into every request's slot, dasc_refresh of the heads left out, from the
              inputs of the prefix's last tokens
  prompt      dasc_linear_attn over the requests' own tokens, ragged, states in place
  score       dasc_linear_attn over [last token, drafts] of every request, no destination
  verify      dasc_verify_drafts on the stack's probabilities against the draft model's
  commit      dasc_linear_attn without an output over the same rows, lens = n_emitted

Every layer is  h = norm(x) -> projections -> linear attention -> norm of each head with a gate ->
projection -> x + norm(.),  the norms by dasc_block_norm: the one after a block also gives the next
block's input.

    python examples/speculative_gdn.py --requests 8 --steps 8 --drafts 4
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


class Stack:
    """`layers` GDN blocks between an embedding and a head, weights from `seed`."""

    def __init__(self, layers=4, heads=8, qk_heads=4, dk=128, dv=128, width=512, vocab=4096, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)

        def w(*size):
            return (torch.randn(size, generator=gen, device="cuda") / size[0] ** 0.5).to(BF16)

        self.shape = D.Shape("gdn", layers, heads, qk_heads, dk, dv)
        self.width, self.vocab, self.scale = width, vocab, dk ** -0.5
        self.embed = torch.randn(vocab, width, generator=gen, device="cuda").to(BF16)
        self.head = w(width, vocab)
        self.bigram = w(width, vocab)            # the draft model: the last token alone
        self.first = torch.ones(width, device="cuda", dtype=BF16)
        self.blocks = []
        # decays from a few tokens to many thousands, as trained heads have them
        self.log_decay = np.tile(-np.geomspace(1e-4, 0.6, heads), (layers, 1))
        for i in range(layers):
            self.blocks.append(dict(
                qk=w(width, 2 * qk_heads * dk), v=w(width, heads * dv), z=w(width, heads * dv),
                gb=w(width, 2 * heads), o=w(heads * dv, width),
                g=torch.tensor(self.log_decay[i], device="cuda", dtype=F32),
                head_norm=torch.ones(dv, device="cuda", dtype=BF16),
                post=torch.full((width,), 0.5, device="cuda", dtype=BF16), next=self.first.clone()))

    def inputs(self, b, h):
        """q, k, v, z, g, beta of block b for the rows of h."""
        s = self.shape
        n = h.shape[0]
        qk = F.normalize((h @ b["qk"]).view(n, 2, s.n_qk_heads, s.dk).float(), dim=-1).to(BF16)
        gb = (h @ b["gb"]).float().view(n, 2, s.n_heads)
        g = b["g"] * (0.5 + torch.sigmoid(gb[:, 0]))
        return (qk[:, 0], qk[:, 1], (h @ b["v"]).view(n, s.n_heads, s.dv),
                (h @ b["z"]).view(n, s.n_heads, s.dv), g, torch.sigmoid(gb[:, 1]))

    def forward(self, tokens, states, src, dst, cu, max_len, rows=None):
        """Runs the rows through every layer.  Returns the probabilities after the rows named by
        `rows` (all if None) and, for each layer, the inputs of its states."""
        s = self.shape
        x = self.embed[tokens]
        h = torch.empty_like(x)
        D.dasc_block_norm(x, w_post=self.first, x_out=h)
        kept = []
        for layer, b in enumerate(self.blocks):
            q, k, v, z, g, beta = self.inputs(b, h)
            o = torch.empty_like(v)
            D.dasc_linear_attn(s, layer, states, src, dst, q, k, v, g, o, cu, max_len, beta=beta,
                               scale=self.scale)
            D.dasc_block_norm(o, gate=z, act="silu", w_post=b["head_norm"], x_out=o)
            y = o.view(-1, s.n_heads * s.dv) @ b["o"]
            D.dasc_block_norm(y, w_post=b["post"], x=x, w_pre=b["next"], x_out=x, h_out=h)
            kept.append((k, v, g, beta))
        h = h if rows is None else h[rows]
        return torch.softmax((h @ self.head).float(), -1), kept

    def draft(self, tokens, m, gen):
        """m tokens for each request from the bigram, and the probabilities that they were drawn with."""
        n = tokens.numel()
        drawn = torch.empty(n, m, dtype=I32, device="cuda")
        probs = torch.empty(n, m, self.vocab, device="cuda")
        for i in range(m):
            probs[:, i] = torch.softmax((self.embed[tokens] @ self.bigram).float(), -1)
            tokens = torch.multinomial(probs[:, i], 1, generator=gen)[:, 0]
            drawn[:, i] = tokens
        return drawn, probs


def i32(a):
    return torch.tensor(a, dtype=I32, device="cuda")


def hit(model, states, prefix, slots, window=16):
    """The prefix's state, by way of its checkpoint, in every slot of `slots`."""
    s = model.shape
    plan = D.dasc_plan(s, model.log_decay.reshape(-1), "threshold", w_max=window)
    n = prefix.numel()
    _, kept = model.forward(prefix, states, None, i32([0]), i32([0, n]), n, rows=[n - 1])
    ckpt = torch.empty(1, max(1, plan["n_rows"]), s.dv, device="cuda")
    rows = i32(plan["unit_row"])
    D.dasc_pack(s, states, i32([0]), rows, ckpt, i32([0]))
    states.fill_(float("nan"))                   # nothing but the checkpoint is left
    inv, where = i32(plan["inv_row"]), i32(slots)
    D.dasc_restore(s, ckpt, i32([0] * len(slots)), inv, states, where, plan["n_rows"])
    W = min(window, n)
    for layer, (k, v, g, beta) in enumerate(kept):
        tail = [t[n - W:].transpose(0, 1).expand(len(slots), *t.shape[1:2], W, *t.shape[2:]).contiguous()
                for t in (k, v, g, beta)]
        D.dasc_refresh(s, layer, inv, states, where, *tail, W)
    return plan


def serve(model, requests=8, prefix=200, prompts=(1, 90), steps=8, drafts=4, seed=1, log=None):
    """Emits tokens for every request.  Returns the list of each request's tokens and the number
    accepted in every step; `log`, a list, receives layer 0's states' start and what each commit took."""
    gen = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = model.shape
    slots = [int(x) for x in 1 + rng.permutation(requests)]
    states = torch.empty(requests + 1, s.n_layers, s.n_heads, s.dk, s.dv, device="cuda")
    hit(model, states, torch.randint(model.vocab, (prefix,), generator=gen, device="cuda"), slots)
    slot = i32(slots)
    if log is not None:
        log.append((slots, states[:, 0].clone()))

    # the prompts: all but the last token go into the states, the last opens the first step
    lens = rng.integers(prompts[0], prompts[1] + 1, requests)
    tokens = torch.randint(model.vocab, (int(lens.sum()),), generator=gen, device="cuda")
    cu = i32(np.concatenate([[0], np.cumsum(lens)]))
    _, kept = model.forward(tokens, states, slot, slot, cu, int(lens.max()), rows=[0])
    if log is not None:
        log.append((kept[0], cu.tolist(), lens.tolist()))
    last = torch.randint(model.vocab, (requests,), generator=gen, device="cuda")

    rows = drafts + 1
    cu = i32(np.arange(requests + 1) * rows)
    out = torch.empty(requests, rows, dtype=I32, device="cuda")
    n_emitted = torch.empty(requests, dtype=I32, device="cuda")
    emitted, accepted = [[] for _ in range(requests)], []
    for _ in range(steps):
        drawn, q = model.draft(last, drafts, gen)
        tokens = torch.cat([last[:, None], drawn.long()], 1).reshape(-1)
        p, kept = model.forward(tokens, states, slot, None, cu, rows)
        D.dasc_verify_drafts(p.view(requests, rows, -1), drawn,
                             torch.rand(requests, drafts, generator=gen, device="cuda"),
                             torch.rand(requests, generator=gen, device="cuda"), out, n_emitted, draft=q)
        for layer, (k, v, g, beta) in enumerate(kept):
            D.dasc_linear_attn(s, layer, states, slot, slot, None, k, v, g, None, cu, rows, beta=beta,
                               lens=n_emitted, scale=model.scale)
        # the host needs the tokens for its clients; the next step only the last of them, on the device
        last = out.gather(1, (n_emitted - 1).long()[:, None])[:, 0].long()
        counts = n_emitted.tolist()
        for r, ids in enumerate(out.tolist()):
            emitted[r] += ids[:counts[r]]
        accepted.append(sum(counts) - requests)
        if log is not None:
            log.append((kept[0], cu.tolist(), counts))
    if log is not None:
        log.append(states[:, 0].clone())
    return emitted, accepted


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    model = Stack(layers=a.layers)
    serve(model, a.requests, steps=1, drafts=a.drafts)         # the first calls load the kernels
    torch.cuda.synchronize()
    t = time.perf_counter()
    emitted, accepted = serve(model, a.requests, steps=a.steps, drafts=a.drafts)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    n = sum(map(len, emitted))
    print(f"{a.requests} requests, {a.steps} steps of {a.drafts} drafts: {n} tokens, "
          f"{sum(accepted) / (a.requests * a.steps):.2f} drafts accepted a step, {1e3 * t:.1f} ms in all")


if __name__ == "__main__":
    main()

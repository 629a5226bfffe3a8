"""The beam example, end to end (GPU): every beam that it returns must be what the model gives for its tokens.

The search keeps states and pages through forks and reorderings; the check runs each returned sequence alone, prompt
and tokens in one call, from nothing.  Both go through bf16 layers in another order of summation (a prompt's chunks
against single tokens), so a log-probability differs by the layers' rounding: each of the at most eight roundings to
bf16 of a layer, 2^-9 relative, moves the residual by at most that, and the head's logits have a deviation of about
1 over `width` terms, so 4 layers x 8 x 2^-9 = 2^-4 bounds a logit's shift by far, and a score's of `steps`
tokens by twice that for each token (its logit and its log-sum).  A state or page of another beam shifts logits by
their own size, about 1.
"""

import numpy as np
import pytest

from examples import beam_hybrid as E
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu


def alone(model, tokens, prompt, page=16):
    """Log-probabilities of tokens[prompt:] after all before them."""
    import torch

    T = tokens.numel()
    width = -(-T // page)
    s = model.shape
    cache = torch.zeros(width, model.n_attn, 2, page, model.kv_heads, model.d, dtype=torch.bfloat16, device="cuda")
    states = torch.zeros(1, s.n_layers, s.n_heads, s.dk, s.dv, device="cuda")
    pos = torch.arange(T, device="cuda")
    table = torch.arange(width, device="cuda").int()[None]
    logits = model.forward(tokens, pos.int(), E.i32([0, T]), T, states, E.i32([0]), cache, table, E.i32([T]), pos,
                           slice(None))
    logp = torch.log_softmax(logits, -1)
    return logp[prompt - 1:-1].gather(1, tokens[prompt:, None])[:, 0]


@pytest.mark.parametrize("lens,beams,steps", [((1, 16, 33), 3, 20), ((50,), 5, 18), ((15, 31), 1, 4)])
def test_beams_are_what_the_model_gives(lens, beams, steps):
    import torch

    announce(f"beam example: prompts {lens}, {beams} beams, {steps} steps")
    model = E.Hybrid()
    gen = torch.Generator("cuda").manual_seed(3)
    prompts = [torch.randint(model.vocab, (k,), generator=gen, device="cuda") for k in lens]
    out, scores = E.search(model, prompts, beams, steps)
    torch.cuda.synchronize()
    assert out.shape == (len(lens), beams, steps) and (out >= 0).all() and (out < model.vocab).all()
    got = scores.cpu().numpy()
    assert np.isfinite(got).all() and (np.diff(got, axis=1) <= 0).all()
    for r, p in enumerate(prompts):
        assert len({tuple(b.tolist()) for b in out[r]}) == beams
        for b in range(beams):
            want = alone(model, torch.cat([p, out[r, b].long()]), len(p)).sum().item()
            assert abs(got[r, b] - want) <= 2 * steps * 2.0 ** -4, (r, b, got[r, b], want)

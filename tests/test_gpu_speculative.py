"""The speculative serving example, end to end (GPU): what its steps leave in the states.

A request's state of layer 0 after all steps must be the recurrence in 64 bits over the rows that
were kept of every step, from the state that the prefix hit left: scored drafts that were rejected
leave no trace.  Tolerance as for the operator itself, for the number of tokens taken: states go
by 2^-24 (16 + 4 sqrt(T)) of their norm for each call, of which there are as many as steps.
"""

import math

import numpy as np
import pytest

from examples import speculative_gdn as E
from oracle import operators as OO
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,prompts,steps,drafts", [(3, (1, 70), 3, 4), (2, (5, 5), 2, 0), (5, (1, 9), 2, 10)])
def test_states_hold_the_kept_tokens(requests, prompts, steps, drafts):
    import torch

    announce(f"speculative example: {requests} requests, {steps} steps of {drafts} drafts")
    model = E.Stack(layers=2, heads=4, qk_heads=2, dk=64, dv=64, width=128, vocab=600)
    log = []
    emitted, accepted = E.serve(model, requests, 40, prompts, steps, drafts, log=log)
    torch.cuda.synchronize()
    assert all(steps <= len(x) <= steps * (drafts + 1) for x in emitted)
    assert all(0 <= t < model.vocab for x in emitted for t in x)
    assert sum(map(len, emitted)) == sum(accepted) + requests * steps
    assert drafts == 0 or sum(accepted) > 0
    (slots, start), calls, last = log[0], log[1:-1], log[-1]
    for r, slot in enumerate(slots):
        S = start[slot].cpu().double().numpy()
        assert np.isfinite(S).all()
        for kept, cu, counts in calls:
            k, v, g, beta = (t[cu[r]:cu[r] + counts[r]].cpu().double().numpy() for t in kept)
            _, S, _ = OO.linear_attn(S, k, k, v, g, beta, 1.0)
        tokens = sum(c[r] for _, _, c in calls)
        tol = 2.0 ** -24 * (16 * len(calls) + 4 * math.sqrt(tokens))
        got = last[slot].cpu().double().numpy()
        for h in range(len(S)):
            e = np.linalg.norm(got[h] - S[h])
            assert e <= tol * np.linalg.norm(S[h]), (r, h, e / np.linalg.norm(S[h]), tol)

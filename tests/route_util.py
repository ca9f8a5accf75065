"""Choices of experts of many tokens that repeat a few rows, against the oracle on those rows."""
import numpy as np
import torch

from oracle import expert_reference as ex
from test_gpu_experts import route, up

# Weights are formed in 64 bits and rounded once: half a step of float32, and 2^-44 for what comes before
WEIGHT = 2.0 ** -24 * (1 + 2.0 ** -20)


def check_repeated(ctx, rows, tokens, bias, score, groups, top_groups, best, k, renorm, scale, mask=None, weight=WEIGHT):
    """rows [r, experts] float32 or bf16 on the device, token t has row t % r; mask [tokens] uint8."""
    r = rows.shape[0]
    logits = rows.repeat(-(-tokens // r), 1)[:tokens].contiguous()
    got_e, got_w = route(ctx, logits, None if bias is None else up(bias), None if mask is None else up(mask), score, groups, top_groups, best, k, renorm, scale)
    want_e, want_w = ex.route(rows[:tokens].cpu().double().numpy(), bias, None, score, groups, top_groups, best, k, renorm, scale)
    of = np.arange(tokens) % r
    want_e, want_w = want_e[of], want_w[of]
    if mask is not None:
        want_e[mask == 0], want_w[mask == 0] = -1, 0.0
    assert np.array_equal(got_e, want_e), (np.argwhere(got_e != want_e)[:5], got_e[(got_e != want_e).any(axis=1)][:1], want_e[(got_e != want_e).any(axis=1)][:1])
    assert np.all(np.abs(got_w - want_w) <= weight * np.abs(want_w) + 2.0 ** -150)

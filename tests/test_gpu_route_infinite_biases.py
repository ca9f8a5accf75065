"""Biases of +infinity: their experts come first, of several the lowest, however many tokens share a wave."""
import numpy as np
import pytest
import torch

from paper_2510_25590_amd import binding as rg
from route_util import check_repeated
from test_gpu_experts import up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


@pytest.mark.parametrize("tokens", [5, 8191, 8192, 8195])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts,groups,top_groups,best,k", [(8, 1, 1, 1, 2), (8, 1, 1, 1, 8), (64, 1, 1, 1, 6), (128, 1, 1, 1, 14), (256, 8, 3, 2, 8), (250, 5, 2, 1, 7), (256, 16, 3, 2, 9)])
def test_infinite_biases(ctx, experts, groups, top_groups, best, k, dtype, score, tokens):
    rng = np.random.default_rng(experts + k)
    rows = rng.normal(size=(7, experts)).astype(np.float32)
    rows[1, experts // 2] = -np.inf
    rows[2, :] = 0.25
    rows[3, experts - 1] = np.nan
    rows = up(rows).to(dtype)
    for forced in ([2], [experts - 1], [1, experts // 2], [0, 1, 2, 3], list(range(experts)), []):
        bias = (0.1 * rng.normal(size=experts)).astype(np.float32)
        bias[forced] = np.inf
        if experts // 3 not in forced:
            bias[experts // 3] = -np.inf
        check_repeated(ctx, rows, tokens, bias, score, groups, top_groups, best, k, True, 1.0)

"""The choice of experts on both sides of the numbers of tokens from which four share a wave (2048, with a bias or groups 8192), of choices (14) and of groups (16) up to which they do."""
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


def normal_rows(rng, experts, dtype):
    return up(rng.normal(size=(37, experts)) * 1.5, torch.float32).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k", [(1, 1), (8, 2), (60, 4), (64, 6), (65, 8), (128, 14), (128, 15), (160, 8), (256, 14), (256, 15), (257, 3)])
def test_by_logits_alone(ctx, experts, k, score, dtype):
    """64, 128 and 256 experts: 4, 8 and 16 of them to a lane, whole pieces; others by elements; 257: a wave to a token."""
    rng = np.random.default_rng(experts + k)
    rows = normal_rows(rng, experts, dtype)
    for tokens in (2047, 2048, 2049):
        check_repeated(ctx, rows, tokens, None, score, 1, 1, 1, k, True, 2.5, mask=None if tokens == 2049 else (rng.random(tokens) < 0.7).astype(np.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("use_bias", [False, True])
@pytest.mark.parametrize("experts,groups,top_groups,best,k", [(60, 1, 1, 1, 4), (64, 2, 1, 2, 6), (256, 1, 1, 1, 14), (128, 4, 2, 2, 14), (128, 4, 2, 2, 15), (160, 8, 3, 1, 6), (256, 8, 4, 2, 8), (72, 9, 4, 2, 5),
                                                              (256, 16, 5, 2, 9), (16, 16, 3, 2, 3), (240, 15, 15, 1, 13), (68, 17, 5, 1, 8), (333, 3, 2, 2, 7)])
def test_by_scores(ctx, experts, groups, top_groups, best, k, use_bias, score, dtype):
    """(groups 1 without a bias is the choice by logits again, at more tokens)"""
    rng = np.random.default_rng(experts + groups + k)
    rows = normal_rows(rng, experts, dtype)
    bias = (0.2 * rng.normal(size=experts)).astype(np.float32) if use_bias else None
    for tokens in (8191, 8192, 8195):
        check_repeated(ctx, rows, tokens, bias, score, groups, top_groups, best, k, True, 2.5, mask=None if tokens == 8195 else (rng.random(tokens) < 0.7).astype(np.uint8))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top_groups,best", [(1, 1, 1), (4, 2, 2), (4, 2, 1)])
@pytest.mark.parametrize("use_bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_values(ctx, dtype, use_bias, groups, top_groups, best, score):
    """Ties, NaN, infinities, the largest and smallest values, fewer experts than are asked for; a bias that takes experts out."""
    e, k = 24, 6
    rng = np.random.default_rng(3)
    l = rng.normal(size=(17, e)).astype(np.float32)
    l[0] = 0.0
    l[1] = -np.inf
    l[2] = np.nan
    l[3], l[3, 7] = -np.inf, 1.0
    l[4, ::2] = np.nan
    l[5, 3], l[5, 11] = np.inf, np.inf
    l[6] = 3.0e38 * np.sign(l[6])
    l[7] *= 40.0
    l[8] = -200.0 - np.arange(e)
    l[9] = 1e-30 * np.arange(e)
    l[10, 6:] = -np.inf
    l[11] = np.round(l[11])
    l[12] = -0.0
    l[12, ::3] = 0.0
    l[13] = 88.0 + np.arange(e) % 5
    l[14] = -1.0e4
    l[15, :18] = -np.inf
    bias = None
    if use_bias:
        bias = (0.3 * rng.normal(size=e)).astype(np.float32)
        bias[5], bias[9], bias[20] = -np.inf, np.nan, 4.0
    for tokens in (2049, 8195):
        check_repeated(ctx, up(l).to(dtype), tokens, bias, score, groups, top_groups, best, k, True, 1.0)


@pytest.mark.parametrize("score,groups,top_groups,best,renorm", [("sigmoid", 1, 1, 1, True), ("softmax", 8, 3, 2, False)])
def test_near_ties(ctx, score, groups, top_groups, best, renorm):
    """Scores of neighbouring float32 logits with a bias of one value, beside tokens that are sure."""
    base = np.float32(1.0)
    l = np.full((9, 64), base, np.float32)
    for t in range(8):
        l[t, 10 + t] = np.nextafter(base, np.float32(2.0))
        l[t, 40 - t] = np.nextafter(base, np.float32(0.0))
    l[8] = np.linspace(-3.0, 3.0, 64)
    for tokens in (9, 8191, 8192, 8195):
        check_repeated(ctx, up(l), tokens, np.full(64, 3.0, np.float32), score, groups, top_groups, best, 4, renorm, 1.0)
